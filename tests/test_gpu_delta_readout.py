"""The operators of a readout with a matrix for a state, run together: gradients through the whole readout against float64 automatic differentiation, whole sequences against
single frames, and that the example runs."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def features(T, B, F, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.rand(T, B, F, generator=g, device=DEV) < 0.2).to(torch.float32)


def in_64(net, x, lengths, h0):
    """The readout in float64 on the CPU, step by step, from the values that the 8-bit weights stand for.  Returns logits and the leaves."""
    import delta_readout
    T, B = x.shape[:2]
    leaf = lambda t: t.detach().cpu().double().requires_grad_()
    w = {"w_in": leaf(api.tac_dequantize(net.in8["rows"], net.F)), "w_out": leaf(api.tac_dequantize(net.out8["rows"], net.D))}
    w.update({n: leaf(getattr(net, n)) for n in ("b_in", "gain", "gain_q", "gain_k")})
    w.update(x=leaf(x), h0=leaf(h0))
    q, k, v, gate, write = net.parts(w["x"] @ w["w_in"].t() + w["b_in"])
    half = net.dk // 2
    angle = torch.arange(T).double()[:, None] * 10000.0 ** (-torch.arange(half).double() / half)
    c, s = torch.cos(angle)[:, None, None], torch.sin(angle)[:, None, None]

    def head(t, gain):
        t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + delta_readout.EPS) * gain
        return torch.cat([t[..., :half] * c - t[..., half:] * s, t[..., half:] * c + t[..., :half] * s], -1)
    share = net.hv // net.hk
    q, k = (head(t, w[n]).repeat_interleave(share, 2) for t, n in ((q, "gain_q"), (k, "gain_k")))
    a, b, S, outs = torch.sigmoid(gate), torch.sigmoid(write), w["h0"], []
    for t in range(T):
        on = (t < torch.tensor(lengths)).double()[:, None, None]
        faded = a[t][..., None, None] * S
        u = b[t][..., None] * (v[t] - (faded * k[t][..., None]).sum(2))
        new = faded + k[t][..., None] * u[..., None, :]
        outs.append((new * q[t][..., None]).sum(2) * on)
        S = on[..., None] * new + (1 - on[..., None]) * S
    o = torch.stack(outs).flatten(2)
    y = o * torch.rsqrt((o * o).mean(-1, keepdim=True) + delta_readout.EPS) * w["gain"]
    return y @ w["w_out"].t(), w


def test_gradients_of_the_readout_against_automatic_differentiation():
    import delta_readout
    T, B, F = 70, 4, 160
    net = delta_readout.DeltaReadout(F, 2, 4, 32, 24, 7, dtype=torch.float32, seed=3)
    net.lay_out()
    g = torch.Generator(device=DEV).manual_seed(4)
    x, lengths = features(T, B, F, 5), [70, 66, 40, 64]
    h0 = torch.randn(B, 4, 32, 24, generator=g, device=DEV) / 6
    on = (torch.arange(T, device=DEV)[:, None] < torch.tensor(lengths, device=DEV))[..., None]
    grad = torch.randn(T, B, 7, generator=g, device=DEV) * on                  # logits behind a length are nobody's
    logits, _, kept = net.forward(x, torch.tensor(lengths, dtype=torch.int32, device=DEV), h0)
    got = net.backward(kept, grad)
    want, w = in_64(net, x, lengths, h0)
    want.backward(grad.cpu().double())
    # y, the logits' gradients and the rows' gradients are rounded to 8 bits, 2^-4 of each at most; a result's rounding errors have mixed signs, so that its 2-norm is
    # off by less than 2^-4 of what it is made of: two such roundings behind one another here
    pairs = [("logits", logits, want)] + [(n, got[n].view(w[n].shape), w[n].grad) for n in ("w_in", "w_out", "b_in", "gain", "gain_q", "gain_k", "x", "h0")]
    for name, mine, exact in pairs:
        off = float(((mine.cpu().double() - exact).norm() / exact.norm()).detach())
        assert off < 2 * 2 ** -4, (name, off)


def test_frame_by_frame_gives_the_sequences_answers():
    import delta_readout
    T, B, F = 90, 6, 128
    net = delta_readout.DeltaReadout(F, 2, 4, 64, 48, 5, seed=6)
    net.lay_out()
    x = features(T, B, F, 7)
    whole, last, _ = net.forward(x)
    g = torch.Generator(device=DEV).manual_seed(8)
    pool = torch.zeros(B + 3, 4, 64, 48, device=DEV)
    slots = torch.randperm(B + 3, generator=g, device=DEV)[:B].to(torch.int32)
    times = lambda t: torch.full((B,), t, dtype=torch.int32, device=DEV)
    running = torch.stack([net.step(x[t], times(t), pool, slots) for t in range(T)])
    # the same products in another order and, where that moves a bfloat16 number to its neighbour, 2^-8 of it and an 8-bit step (2^-4) of single features among 192,
    # whose signs are mixed
    assert float((running - whole).abs().max() / whole.abs().max()) < 2 ** -4
    # states are float32 from the same bfloat16 rows: 64 roundings of 2^-24 in the 2-norm
    assert float((pool[slots.long()] - last).norm() / last.norm()) < 64 * 2 ** -24
    # a prompt in one call, then frames
    first = net.forward(x[:50])
    pool[slots.long()] = first[1]
    rest = torch.stack([net.step(x[t], times(t), pool, slots) for t in range(50, T)])
    assert float((rest - whole[50:]).abs().max() / whole.abs().max()) < 2 ** -4


def test_a_training_step_captured_and_replayed():
    import delta_readout
    T, B, F = 70, 3, 128
    net = delta_readout.DeltaReadout(F, 1, 2, 32, 32, 5, seed=9)
    net.lay_out()
    x, grad = features(T, B, F, 10), torch.ones(T, B, 5, device=DEV)

    def call():
        logits, last, kept = net.forward(x)
        return {"logits": logits, "last": last, **net.backward(kept, grad, want_bias=False)}
    want = {n: t.clone() for n, t in call().items()}
    from delta_util import captured
    for r in captured(call):
        assert all(torch.equal(r[n], want[n]) for n in want)
        call()


def test_the_example_runs():
    import delta_readout
    losses = delta_readout.main(steps=6)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses)
