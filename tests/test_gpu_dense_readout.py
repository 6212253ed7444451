"""The example that runs the dense operators together: training through the spiking layer, then frame by frame; and its gradients against
float64 automatic differentiation."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_training_lowers_the_loss_and_frames_give_the_sequences_answers():
    import dense_readout
    losses, right, apart = dense_readout.main()
    # five classes: ln 5 = 1.61 at the start; classes differ in the rates of 256 pixels, which a trained readout tells apart
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0] and right > 0.8
    # the same products in another order and, where that moves a bfloat16 number to its neighbour, 2^-8 of it and an 8-bit step (2^-4) of
    # single features among 128, whose signs are mixed
    assert apart < 2 ** -4


def test_gradients_of_the_readout_against_automatic_differentiation():
    import dense_readout
    T, B, F, D, classes = 40, 6, 200, 96, 7
    net = dense_readout.DenseReadout(F, D, classes, dtype=torch.float32, seed=3)
    net.lay_out()
    g = torch.Generator(device=DEV).manual_seed(4)
    spikes = (torch.rand(T, B, F, generator=g, device=DEV) < 0.2).to(torch.uint8)
    grad = torch.randn(T, B, classes, generator=g, device=DEV)
    logits, _, kept = net.forward(spikes)
    got = net.backward(kept, grad)

    from paper_2603_13810_amd import api
    w_in, w_out = (api.tac_dequantize(q["rows"], k).cpu().double().requires_grad_() for q, k in ((net.in8, F), (net.out8, D)))
    b_in, gain = net.b_in.cpu().double().requires_grad_(), net.gain.cpu().double().requires_grad_()
    x = spikes.cpu().double().requires_grad_()
    both = x @ w_in.t() + b_in
    a, u, h, outs = torch.sigmoid(both[..., :D]), both[..., D:], torch.zeros(B, D, dtype=torch.float64), []
    for t in range(T):
        h = a[t] * h + (1 - a[t]) * u[t]
        outs.append(h)
    s = torch.stack(outs) + u
    y = s * torch.rsqrt((s * s).mean(2, keepdim=True) + dense_readout.EPS) * gain
    want = y @ w_out.t()
    want.backward(grad.cpu().double())
    # y, the logits' gradients and the gates' and values' gradients are rounded to 8 bits, 2^-4 of each at most; a result's rounding errors
    # have mixed signs, so that its 2-norm is off by less than 2^-4 of what it is made of: two such roundings behind one another here
    for name, mine, exact in [("logits", logits, want), ("w_in", got["w_in"], w_in.grad), ("w_out", got["w_out"], w_out.grad),
                              ("b_in", got["b_in"], b_in.grad), ("gain", got["gain"], gain.grad), ("spikes", got["spikes"].view(T, B, F), x.grad)]:
        off = float(((mine.cpu().double() - exact).norm() / exact.norm()).detach())
        assert off < 2 * 2 ** -4, (name, off)
