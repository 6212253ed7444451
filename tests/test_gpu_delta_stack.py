"""A spiking layer in front of a readout with a matrix for a state: whole sequences of frames against frame by frame with the membranes and the states carried, and a
training step down to the layer's weights."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, B, SIDE, CHANNELS, CLASSES = 70, 6, 16, 8, 5


def network():
    import delta_readout
    import dense_readout
    net = dense_readout.Network(SIDE, CHANNELS, 32, CLASSES, device=DEV)
    readout = delta_readout.DeltaReadout(CHANNELS * net.out_side ** 2, 2, 4, 32, 24, CLASSES, seed=4)
    readout.lay_out()
    frames = (torch.rand(T, B, 1, SIDE, SIDE, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV) < 0.3).to(torch.uint8)
    return net, readout, frames


def test_frames_one_by_one():
    net, readout, frames = network()
    spikes = net.spikes_of(frames)[0]
    assert 0.01 < float(spikes.float().mean()) < 0.99
    whole, last, _ = readout.forward(spikes)
    v = torch.zeros(B, CHANNELS, net.out_side, net.out_side, device=DEV)
    pool = torch.zeros(B + 2, 4, 32, 24, device=DEV)
    slots = torch.tensor([7, 0, 3, 1, 6, 4], dtype=torch.int32, device=DEV)
    running = []
    for t in range(T):
        now = net.spikes_of(frames[t:t + 1], v)[0]
        assert torch.equal(now[0], spikes[t])
        running.append(readout.step(now[0], torch.full((B,), t, dtype=torch.int32, device=DEV), pool, slots))
    # products in another order: where that moves a bfloat16 number to its neighbour, 2^-8 of it and an 8-bit step (2^-4) of single features among 96, whose signs are mixed
    assert float((torch.stack(running) - whole).abs().max() / whole.abs().max()) < 2 ** -4
    # states are float32 from the same bfloat16 rows: 64 roundings of 2^-24 in the 2-norm
    assert float((pool[slots.long()] - last).norm() / last.norm()) < 64 * 2 ** -24


def test_a_training_step_down_to_the_layers_weights():
    net, readout, frames = network()

    def step():
        spikes, (stack, packed, layer) = net.spikes_of(frames, trace=True)
        logits, _, kept = readout.forward(spikes)
        grad = torch.softmax(logits, 2) / T
        grads = readout.backward(kept, grad)
        grad_spikes = grads["x"].view(T, B, CHANNELS, net.out_side, net.out_side)
        return grads, grad_spikes, api.tac_stack_backward(stack, [net.w_conv], packed, grad_spikes, alpha=5.0)[0]["grad_w"]
    grads, grad_spikes, grad_w = step()
    assert grad_w.shape == net.w_conv.shape and all(torch.isfinite(t).all() for t in grads.values()) and float(grad_w.abs().max()) > 0
    # the readout's gradients, what it hands back to the layer among them, are the same bits again; the layer's own sums use atomics, in any order
    again, again_spikes, _ = step()
    assert all(torch.equal(grads[n], again[n]) for n in grads if n != "b_in") and torch.equal(grad_spikes, again_spikes)
