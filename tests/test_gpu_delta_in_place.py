"""The gated delta rule through the C interface where an output takes an input's place, which the Python calls leave no way to: last states on the first ones, the
first states' gradient on the last ones'; the same bits as with places of their own, and from call to call.  And the walk over wide tiles without kept states."""
import ctypes

import numpy as np
import pytest
import torch

import delta_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("query", "key", "value", "gate", "write")
TYPES = [torch.float32, torch.bfloat16]


def describe(x, T, B, hk, hv, dk, dv):
    s = lambda t: api.tac_delta_strides_t(*(list(t.stride()) + [1])[:3])
    d = api.tac_delta_desc_t(T=T, B=B, k_heads=hk, v_heads=hv, Dk=dk, Dv=dv, dtype=api.TAC_BF16 if x["key"].dtype == torch.bfloat16 else api.TAC_FP32)
    for n in NAMES:
        setattr(d, n, s(x[n]))
        setattr(d, "grad_" + n, s(x[n]))
    d.out = s(x["value"])
    return d


def at(t):
    return None if t is None else t.data_ptr()


def scan(d, x, lengths, h0, out, h_last, states, updates):
    work = torch.empty(api.lib().tac_delta_scan_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    assert api.lib().tac_delta_scan(ctypes.byref(d), *[at(x[n]) for n in NAMES], at(lengths), at(h0), at(out), at(h_last), at(states), at(updates), at(work), stream) == 0
    torch.cuda.synchronize()


def backward(d, x, lengths, states, updates, grad_out, grad_last, grads, grad_h0):
    work = torch.empty(api.lib().tac_delta_scan_backward_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    assert api.lib().tac_delta_scan_backward(ctypes.byref(d), *[at(x[n]) for n in NAMES], at(lengths), at(states), at(updates), at(grad_out), at(grad_last),
                                             *[at(g) for g in grads], at(grad_h0), at(work), stream) == 0
    torch.cuda.synchronize()


# several tiles of columns, of 16 and (the last two) of 32
SHAPES = [(150, 4, 2, 4, 64, 100), (70, 3, 1, 2, 128, 40), (200, 2, 1, 1, 33, 17), (70, 16, 16, 32, 40, 24), (66, 16, 16, 16, 128, 80)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("T,B,hk,hv,dk,dv", SHAPES)
def test_states_in_place(T, B, hk, hv, dk, dv, kept, dtype):
    x, h0 = O.delta_inputs(T, B, hk, hv, dk, dv, dtype, 200 + T)
    lengths = torch.tensor([0, T, T // 2, 64][:B] + [1 + 3 * b for b in range(4, B)], dtype=torch.int32, device=DEV)
    args, d = [x[n] for n in NAMES], describe(x, T, B, hk, hv, dk, dv)
    want = api.tac_delta_scan(*args, lengths=lengths, h0=h0, want_kept=True)
    assert torch.equal(want["h_last"][0], h0[0])
    again = api.tac_delta_scan(*args, lengths=lengths, h0=h0, want_kept=True)
    live = [torch.nonzero(lengths > 64 * c).flatten() for c in range(want["states"].shape[0])]      # of the others nothing is written
    assert torch.equal(again["out"], want["out"]) and torch.equal(again["h_last"], want["h_last"])
    assert all(torch.equal(again["states"][c][b], want["states"][c][b]) for c, b in enumerate(live))
    state, out = h0.clone(), torch.full_like(x["value"], 3.0)
    states = torch.zeros_like(want["states"]) if kept else None
    updates = torch.zeros_like(want["updates"]) if kept else None
    scan(d, x, lengths, state, out, state, states, updates)
    assert torch.equal(out, want["out"]) and torch.equal(state, want["h_last"])
    if kept:
        for c, b in enumerate(live):
            assert torch.equal(states[c][b], want["states"][c][b])
            rows = slice(64 * c, min(64 * c + 64, T))
            assert torch.equal(updates[rows][:, b], want["updates"][rows][:, b]) and torch.equal(again["updates"][rows][:, b], want["updates"][rows][:, b])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,hk,hv,dk,dv", SHAPES)
def test_gradients_of_states_in_place(T, B, hk, hv, dk, dv, dtype):
    x, h0 = O.delta_inputs(T, B, hk, hv, dk, dv, dtype, 300 + T)
    lengths = torch.tensor([0, T, T // 2, 64][:B] + [1 + 3 * b for b in range(4, B)], dtype=torch.int32, device=DEV)
    args, d = [x[n] for n in NAMES], describe(x, T, B, hk, hv, dk, dv)
    kept = api.tac_delta_scan(*args, lengths=lengths, h0=h0, want_kept=True)
    g = torch.Generator(device=DEV).manual_seed(7)
    go, last = torch.randn(x["value"].shape, generator=g, device=DEV).to(dtype), torch.randn(h0.shape, generator=g, device=DEV)
    want = api.tac_delta_scan_backward(*args, kept["states"], kept["updates"], go, lengths=lengths, grad_h_last=last)
    assert torch.equal(want["grad_h0"][0], last[0])
    state, grads = last.clone(), [torch.full_like(a, 3.0) for a in args]
    backward(d, x, lengths, kept["states"], kept["updates"], go, state, grads, state)
    assert torch.equal(state, want["grad_h0"]) and all(torch.equal(t, want["grad_" + n]) for t, n in zip(grads, NAMES))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,hk,hv,dk,dv", [(16, 32, 32, 64, 24), (9, 16, 32, 30, 70), (16, 16, 32, 128, 40)])
def test_wide_tiles_without_kept_states(B, hk, hv, dk, dv, dtype):
    """A batch of prompts: enough heads that a workgroup takes 32 columns, and nothing is kept."""
    x, h0 = O.delta_inputs(70, B, hk, hv, dk, dv, dtype, 400 + dk)
    args = [x[n] for n in NAMES]
    lengths = [70 - 5 * b if b % 3 else 70 for b in range(B)]
    got = api.tac_delta_scan(*args, lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV), h0=h0)
    out, S, _ = O.delta(*[O.as64(a) for a in args], lengths=np.array(lengths), h0=O.as64(h0))
    # sums over up to 128 features and 64 steps of products with a relative error of 2^-24 or so, of numbers that come from two or three such sums: 4 sqrt(192)
    # independent roundings in the 2-norm, four times as many, by the root mean square, in the worst of some 10^5 results; then the result's own
    for name, mine, want, half in (("out", got["out"], out, O.HALF[dtype]), ("h_last", got["h_last"], S, 0.0)):
        rms = np.sqrt((want * want).mean())
        off = np.abs(O.as64(mine) - want)
        assert (off <= half * (1 + 1e-6) * np.abs(want) + 256 * O.U * (np.abs(want) + rms)).all(), name
    kept = api.tac_delta_scan(*args, lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV), h0=h0, want_kept=True)
    assert torch.equal(kept["out"], got["out"]) and torch.equal(kept["h_last"], got["h_last"])
