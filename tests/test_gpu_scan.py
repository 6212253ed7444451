"""Gated linear recurrence, its backward pass and its single step against 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import head_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]
SHAPES = [(1, 1, 1), (1, 3, 130), (2, 1, 64), (31, 2, 33), (32, 2, 64), (33, 1, 100), (64, 3, 128), (65, 2, 7), (100, 5, 256), (511, 1, 48),
          (512, 2, 64), (513, 2, 66), (1030, 1, 200), (2500, 3, 40), (5000, 1, 17), (300, 40, 72), (128, 3, 1026), (9000, 1, 512)]


def make(T, B, D, dtype, seed, ragged=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    both = n(T, B, 2 * D)
    both[..., :D] += 6 * torch.rand(D, generator=g, device=DEV)
    both = both.to(dtype)
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        lengths[0] = 0
        if B > 1:
            lengths[1] = T
    return both[..., :D], both[..., D:], lengths, n(B, D), n(T, B, D).to(dtype), n(B, D)


def reference(gate, value, lengths, h0, grad_out=None, grad_last=None):
    g, u = O.as64(gate), O.as64(value)
    n = None if lengths is None else np.clip(lengths.cpu().numpy(), 0, gate.shape[0])
    out, before, last = O.scan(g, u, n, None if h0 is None else O.as64(h0))
    r = dict(out=out, before=before, h_last=last, g=g, u=u, n=n)
    # a's relative error: exp's argument rounded (|gate| u), exp and 1/x (4 u); the update: 4 u.  Each step's error is at most that
    # of the largest |h| or |value| and shrinks by a: summed over min(T, 1 / (1 - a)) steps
    a = 1.0 / (1.0 + np.exp(-g))
    steps = np.minimum(gate.shape[0], 1.0 / (1.0 - a.max()))
    big = max(np.abs(u).max(), np.abs(before).max(), np.abs(last).max())
    r["tol"] = (16 + 2 * np.abs(g).max()) * O.U * steps * big
    if grad_out is not None:
        go, gl = O.as64(grad_out), None if grad_last is None else O.as64(grad_last)
        r["gg"], r["gv"], r["g0"] = O.scan_backward(g, u, before, go, n, gl)
        # the cotangent obeys the same recurrence backwards and has no (1 - a): up to `steps` gradients of the largest size add up in it
        top = max(np.abs(go).max(), 0 if gl is None else np.abs(gl).max()) * steps
        r["ctol"] = (16 + 2 * np.abs(g).max()) * O.U * steps * top
        r["top"] = top
    return r


def close(got, want, tol, dtype):
    half = O.HALF[dtype]
    assert (np.abs(O.as64(got) - want) <= half * np.abs(want) * (1 + 1e-6) + tol * (1 + half)).all(), np.abs(O.as64(got) - want).max()


def check_forward(r, got, dtype):
    close(got["out"], r["out"], r["tol"], dtype)
    close(got["h_last"], r["h_last"], r["tol"], torch.float32)
    if got["states"] is not None:
        close(got["states"], r["before"][::api.TAC_SCAN_CHUNK], r["tol"], torch.float32)


def check_backward(r, got, dtype):
    big = max(np.abs(r["u"]).max(), np.abs(r["before"]).max())
    close(got["grad_value"], r["gv"], r["ctol"], dtype)
    close(got["grad_gate"], r["gg"], 2 * big * r["ctol"] / 4 + r["top"] * r["tol"] / 4, dtype)
    close(got["grad_h0"], r["g0"], r["ctol"], torch.float32)


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,D", SHAPES)
def test_forward_and_backward(T, B, D, dtype, ragged):
    gate, value, lengths, h0, go, gl = make(T, B, D, dtype, 500 + T, ragged)
    r = reference(gate, value, lengths, h0, go, gl)
    got = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    check_forward(r, got, dtype)
    check_forward(r, api.tac_gated_scan(gate, value, lengths=lengths, h0=h0), dtype)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, lengths=lengths, grad_h_last=gl)
    check_backward(r, back, dtype)
    again = api.tac_gated_scan_backward(gate, value, got["states"], go, lengths=lengths, grad_h_last=gl)
    for k in back:
        assert torch.equal(back[k], again[k])
    if ragged:
        for b, n in enumerate(r["n"]):
            assert not got["out"][n:, b].any() and not back["grad_gate"][n:, b].any() and not back["grad_value"][n:, b].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,D", [(70, 3, 96), (700, 2, 64)])
def test_without_the_optional_tensors(T, B, D, dtype):
    gate, value, _, _, go, _ = make(T, B, D, dtype, 21)
    r = reference(gate, value, None, None, go)
    got = api.tac_gated_scan(gate, value, want_h_last=False, want_states=True)
    assert got["h_last"] is None
    close(got["out"], r["out"], r["tol"], dtype)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, want_grad_h0=False)
    assert back["grad_h0"] is None
    check_backward(r, dict(back, grad_h0=torch.from_numpy(r["g0"])), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["batch_first", "odd_stride", "shifted"])
def test_layouts(dtype, layout):
    T, B, D = 130, 4, 66
    gate, value, lengths, h0, go, gl = make(T, B, D, dtype, 22, ragged=True)
    want = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    want_back = api.tac_gated_scan_backward(gate, value, want["states"], go, lengths=lengths, grad_h_last=gl)
    move = {"batch_first": lambda t: t.transpose(0, 1).contiguous().transpose(0, 1), "odd_stride": lambda t: O.strided(t, 3),
            "shifted": O.shifted}[layout]
    out, gg, gv = (move(torch.zeros_like(go)) for _ in range(3))
    got = api.tac_gated_scan(move(gate), move(value), lengths=lengths, h0=h0, out=out, want_states=True)
    api.tac_gated_scan_backward(move(gate), move(value), got["states"], move(go), lengths=lengths, grad_h_last=gl, grad_gate=gg, grad_value=gv)
    # the same chunks and the same arithmetic, whatever the layout
    for a, b in ((out, want["out"]), (got["h_last"], want["h_last"]), (got["states"], want["states"]), (gg, want_back["grad_gate"]),
                 (gv, want_back["grad_value"])):
        assert torch.allclose(a.float(), b.float(), rtol=2 * O.HALF[dtype], atol=1e-5)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_stands_behind_a_length_is_read_into_nothing(dtype):
    T, B, D = 200, 5, 64
    gate, value, lengths, h0, go, gl = make(T, B, D, dtype, 23, ragged=True)
    clean = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    clean_back = api.tac_gated_scan_backward(gate, value, clean["states"], go, lengths=lengths, grad_h_last=gl)
    behind = (torch.arange(T, device=DEV)[:, None] >= lengths[None, :])[:, :, None]
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        g, u, o = (torch.where(behind, torch.full_like(t, bad), t) for t in (gate, value, go))
        got = api.tac_gated_scan(g, u, lengths=lengths, h0=h0, want_states=True)
        back = api.tac_gated_scan_backward(g, u, got["states"], o, lengths=lengths, grad_h_last=gl)
        for k in ("out", "h_last", "states"):
            assert torch.equal(got[k], clean[k]), k
        for k in back:
            assert torch.equal(back[k], clean_back[k]), k


def test_lengths_outside_the_sequence_are_its_ends():
    gate, value, _, h0, go, gl = make(50, 3, 32, torch.float32, 24)
    wild, tame = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ((-5, 50000, 2 ** 31 - 1), (0, 50, 50)))
    a, b = (api.tac_gated_scan(gate, value, lengths=n, h0=h0, want_states=True) for n in (wild, tame))
    x, y = (api.tac_gated_scan_backward(gate, value, a["states"], go, lengths=n, grad_h_last=gl) for n in (wild, tame))
    assert all(torch.equal(a[k], b[k]) for k in a) and all(torch.equal(x[k], y[k]) for k in x)


@pytest.mark.parametrize("dtype", TYPES)
def test_gates_at_their_ends(dtype):
    T, B, D = 80, 1, 64
    gate, value, _, h0, go, gl = make(T, B, D, dtype, 25)
    gate = gate.clone()
    gate[:, :, 0], gate[:, :, 1], gate[:, :, 2], gate[:, :, 3] = float("inf"), -float("inf"), 200.0, -200.0
    gate[40:, :, 4] = -float("inf")
    value = value.contiguous()
    got = api.tac_gated_scan(gate, value, h0=h0, want_states=True)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, grad_h_last=gl)
    for k in (got, back):
        assert all(torch.isfinite(t).all() for t in k.values())
    for d in (0, 2):
        assert torch.equal(got["out"][:, 0, d], h0[0, d].to(dtype).expand(T))               # nothing leaks
    for d in (1, 3):
        assert torch.equal(got["out"][:, 0, d], value[:, 0, d])                               # nothing is kept
    r = reference(gate[..., 4:], value[..., 4:], None, h0[:, 4:], go[..., 4:], gl[:, 4:])
    close(got["out"][..., 4:], r["out"], r["tol"], dtype)
    close(back["grad_value"][..., 4:], r["gv"], r["ctol"], dtype)


def test_a_sequence_in_pieces_is_the_sequence():
    gate, value, _, h0, _, _ = make(300, 2, 48, torch.float32, 26)
    whole = api.tac_gated_scan(gate, value, h0=h0)
    h, outs = h0, []
    for lo, hi in ((0, 1), (1, 130), (130, 300)):
        r = api.tac_gated_scan(gate[lo:hi], value[lo:hi], h0=h)
        h = r["h_last"]
        outs.append(r["out"])
    assert torch.allclose(torch.cat(outs), whole["out"], rtol=0, atol=2e-5) and torch.allclose(h, whole["h_last"], rtol=0, atol=2e-5)


def test_gradient_against_differences_of_the_kernel():
    T, B, D = 150, 3, 40
    gate, value, lengths, h0, go, gl = make(T, B, D, torch.float32, 27, ragged=True)
    got = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, lengths=lengths, grad_h_last=gl)
    g = torch.Generator(device=DEV).manual_seed(28)
    dg, dv, dh = (torch.randn(*s, generator=g, device=DEV) for s in ((T, B, D), (T, B, D), (B, D)))

    def loss(t):
        o = api.tac_gated_scan(gate + t * dg, value + t * dv, lengths=lengths, h0=h0 + t * dh)
        return float((o["out"].double() * go.double()).sum() + (o["h_last"].double() * gl.double()).sum())
    terms = [(back["grad_gate"] * dg).double(), (back["grad_value"] * dv).double(), (back["grad_h0"] * dh).double()]
    want, size = float(sum(t.sum() for t in terms)), float(sum(t.abs().sum() for t in terms))
    eps = 2.0 ** -7
    # third derivatives: eps^2 = 6e-5 of the terms' size; rounding: 2^-20 of the loss's terms over 2 eps
    assert abs((loss(eps) - loss(-eps)) / (2 * eps) - want) < 1e-3 * size


@pytest.mark.parametrize("T,B,D", [(300, 3, 128), (3000, 1, 64)])
def test_on_another_stream_and_in_a_graph(T, B, D):
    gate, value, lengths, h0, go, gl = make(T, B, D, torch.bfloat16, 29, ragged=True)
    lengths[0] = T
    want = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    want_back = api.tac_gated_scan_backward(gate, value, want["states"], go, lengths=lengths, grad_h_last=gl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True, stream=side.cuda_stream)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, lengths=lengths, grad_h_last=gl, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(back["grad_gate"], want_back["grad_gate"])

    def both():
        o = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
        return o, api.tac_gated_scan_backward(gate, value, o["states"], go, lengths=lengths, grad_h_last=gl)
    for o, b in O.captured(both):
        assert all(torch.equal(o[k], want[k]) for k in o) and all(torch.equal(b[k], want_back[k]) for k in b)
        o["out"].fill_(float("nan"))
        b["grad_gate"].fill_(float("nan"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,D", [(1, 1), (3, 7), (5, 64), (33, 100), (64, 2048), (300, 520)])
def test_single_steps(B, D, dtype):
    g = torch.Generator(device=DEV).manual_seed(30)
    both = torch.randn(B, 2 * D, generator=g, device=DEV).to(dtype)
    gate, value = both[:, :D], both[:, D:]
    pool = torch.randn(B + 5, D, generator=g, device=DEV)
    slots = torch.randperm(B + 5, generator=g, device=DEV)[:B].to(torch.int32)
    r = reference(gate[None], value[None], None, pool[slots.long()])
    before = pool.clone()
    out = api.tac_gated_step(gate, value, pool, slots)
    close(out, r["out"][0], r["tol"], dtype)
    close(pool[slots.long()], r["h_last"], r["tol"], torch.float32)
    left = torch.ones(B + 5, dtype=torch.bool, device=DEV)
    left[slots.long()] = False
    assert torch.equal(pool[left], before[left])
    straight = before[:B].clone()
    r = reference(gate[None], value[None], None, straight)
    close(api.tac_gated_step(gate, value, straight), r["out"][0], r["tol"], dtype)
    close(straight, r["h_last"], r["tol"], torch.float32)


def test_slots_outside_the_pool_touch_nothing():
    B, D = 6, 130
    gate, value, pool = torch.full((B, D), float("nan"), device=DEV), torch.randn(B, D, device=DEV), torch.randn(4, D, device=DEV)
    gate[1] = 0.5
    before = pool.clone()
    slots = torch.tensor([-1, 2, 4, -2 ** 31, 2 ** 31 - 1, 1000], dtype=torch.int32, device=DEV)
    out = api.tac_gated_step(gate, value, pool, slots)
    for b in (0, 2, 3, 4, 5):
        assert not out[b].any()
    assert torch.equal(pool[[0, 1, 3]], before[[0, 1, 3]]) and torch.isfinite(pool).all() and torch.equal(out[1], pool[2])


def test_steps_are_the_scan():
    T, B, D = 40, 3, 96
    gate, value, _, h0, _, _ = make(T, B, D, torch.bfloat16, 31)
    whole = api.tac_gated_scan(gate, value, h0=h0)
    pool = h0.clone()
    outs = [api.tac_gated_step(gate[t], value[t], pool) for t in range(T)]
    assert torch.allclose(pool, whole["h_last"], rtol=0, atol=1e-5)
    assert torch.allclose(torch.stack(outs).float(), whole["out"].float(), rtol=2 ** -7, atol=1e-5)
    steps = torch.zeros(B, D, device=DEV)
    for o in O.captured(lambda: api.tac_gated_step(gate[0], value[0], steps)):
        pass
    want = torch.zeros(B, D, device=DEV)
    for _ in range(4):                                              # once eagerly, three replays
        api.tac_gated_step(gate[0], value[0], want)
    assert torch.equal(steps, want)


def test_offsets_beyond_32_bits():
    T, B, D = 20_000, 60, 1024                                       # 2.4 G elements in each half
    both = torch.empty((T, B, 2 * D), dtype=torch.bfloat16, device=DEV)
    both.normal_()
    gate, value = both[..., :D], both[..., D:]
    got = api.tac_gated_scan(gate, value, want_states=True)
    start = got["states"][-3]
    t0 = (got["states"].shape[0] - 3) * api.TAC_SCAN_CHUNK
    tail = api.tac_gated_scan(gate[t0:], value[t0:], h0=start)
    r = reference(gate[t0:, -1:, :200], value[t0:, -1:, :200], None, start[-1:, :200])
    close(got["out"][t0:, -1:, :200], r["out"], r["tol"], torch.bfloat16)
    assert torch.allclose(got["h_last"], tail["h_last"], rtol=0, atol=1e-4)
    back = api.tac_gated_scan_backward(gate, value, got["states"], got["out"])
    r = reference(gate[t0:, -1:, :200], value[t0:, -1:, :200], None, start[-1:, :200], got["out"][t0:, -1:, :200])
    close(back["grad_value"][t0:, -1:, :200], r["gv"], r["ctol"], torch.bfloat16)


def c_abi(name, T, B, D, dtype, *tensors):
    """The C entry point on contiguous tensors (None: NULL), scratch behind them."""
    d = api.tac_scan_desc_t(T, B, D, B * D, D, B * D, D, B * D, D, api.TAC_BF16 if dtype == torch.bfloat16 else api.TAC_FP32)
    work = torch.empty(max(16, api.lib().tac_gated_scan_workspace_bytes(ctypes.addressof(d))), dtype=torch.uint8, device=DEV)
    status = getattr(api.lib(), name)(ctypes.addressof(d), *(None if t is None else t.data_ptr() for t in tensors), work.data_ptr(),
                                      torch.cuda.current_stream().cuda_stream)
    assert status == api.TAC_OK


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("T,B,D,dtype", [(32768, 1, 2048, torch.bfloat16), (20000, 3, 1000, torch.float32), (9000, 1, 512, torch.float32),
                                         (3001, 2, 65, torch.bfloat16), (100, 3, 96, torch.float32)])
def test_the_last_state_may_take_the_place_of_the_first(T, B, D, dtype, ragged):
    gate, value, lengths, h0, go, gl = (t if t is None else t.contiguous() for t in make(T, B, D, dtype, 32, ragged))
    if ragged and B == 1:
        lengths[0] = T // 3
    want = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    want_back = api.tac_gated_scan_backward(gate, value, want["states"], go, lengths=lengths, grad_h_last=gl)
    state, out, states = h0.clone(), torch.empty_like(go), torch.empty_like(want["states"])
    c_abi("tac_gated_scan", T, B, D, dtype, gate, value, lengths, state, out, state, states)
    assert torch.equal(state, want["h_last"]) and torch.equal(out, want["out"]) and torch.equal(states, want["states"])
    grad, gg, gv = gl.clone(), torch.empty_like(go), torch.empty_like(go)
    c_abi("tac_gated_scan_backward", T, B, D, dtype, gate, value, lengths, states, go, grad, gg, gv, grad)
    assert torch.equal(grad, want_back["grad_h0"]) and torch.equal(gg, want_back["grad_gate"]) and torch.equal(gv, want_back["grad_value"])


def same_ends(got, want, tol, dtype):
    """NaN and infinities of either sign in the same places; the numbers within tol (by channel) and a rounding."""
    got = O.as64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want))
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    ok = np.isfinite(want)
    half = O.HALF[dtype]
    assert (np.abs(got - want)[ok] <= (half * np.abs(want) * (1 + 1e-6) + tol * (1 + half) + 1e-37)[ok]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,D,lengths", [(40, 3, 10, (16, 17, 40)), (40, 3, 11, None), (300, 4, 66, (127, 128, 300, 200)), (3001, 2, 64, (3001, 2000)),
                                           (2500, 1, 12, None), (256, 200, 130, None)])
def test_infinite_states_and_gradients(T, B, D, lengths, dtype):
    g = torch.Generator(device=DEV).manual_seed(33)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    gate, value, h0, go, gl = (n(T, B, D) + 1).to(dtype), n(T, B, D).to(dtype), n(B, D), n(T, B, D).to(dtype), n(B, D)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    args = dict(lengths=lens, h0=h0)
    clean = api.tac_gated_scan(gate, value, want_states=True, **args)
    clean_back = api.tac_gated_scan_backward(gate, value, clean["states"], go, lengths=lens, grad_h_last=gl)
    h0, value, gate, go, gl = h0.clone(), value.clone(), gate.clone(), go.clone(), gl.clone()
    inf, top = float("inf"), torch.finfo(dtype).max
    end = [T] * B if lengths is None else lengths
    h0[:, 0] = inf                                       # an infinite state that is there from the start
    h0[:, 1], gate[:, :, 1] = -inf, -8.0                 # through factors whose product is below float32's smallest
    for b in range(B):
        value[end[b] // 2, b, 2] = inf
        value[end[b] // 3, b, 3], value[end[b] // 2, b, 3] = inf, -inf        # NaN from the second on
        value[end[b] - 1, b, 4] = -inf                   # the last step's
        go[end[b] // 2, b, 6] = inf
        go[end[b] // 2, b, 7], go[end[b] // 3, b, 7] = inf, -inf
    value[::2, :, 5], value[1::2, :, 5] = top, -top      # differences beyond float32, states within it
    gl[:, 8] = -inf
    value[T // 4, :, 9] = float("nan")
    got = api.tac_gated_scan(gate, value, want_states=True, lengths=lens, h0=h0)
    g64, u64, cut = O.as64(gate), O.as64(value), None if lengths is None else np.array(lengths)
    with np.errstate(invalid="ignore"):
        out, before, last = O.scan(g64, u64, cut, O.as64(h0))
        gg, gv, g0 = O.scan_backward(g64, u64, before, O.as64(go), cut, O.as64(gl))
    # as in reference(), by channel: per step (16 + 2 |gate|) roundings of the channel's largest finite value, shrinking by the largest a
    steps = np.minimum(T, 1.0 / (1.0 - 1.0 / (1.0 + np.exp(-g64.max(0)))))
    most = lambda v: np.where(np.isfinite(v), np.abs(v), 0).max(0)
    per = (16 + 2 * np.abs(g64).max(0)) * O.U * steps
    tol = per * np.maximum(np.maximum(most(u64), most(before)), most(last[None]))
    same_ends(got["out"], out, tol, dtype)
    same_ends(got["h_last"], last, tol, torch.float32)
    same_ends(got["states"], before[::api.TAC_SCAN_CHUNK], tol, torch.float32)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, lengths=lens, grad_h_last=gl)
    size = np.maximum(most(O.as64(go)), most(O.as64(gl)[None])) * steps
    same_ends(back["grad_value"], gv, per * size, dtype)
    same_ends(back["grad_h0"], g0, per * size, torch.float32)
    gated = [d for d in range(D) if d != 5]              # h - value itself is beyond float32 there
    wide = 2 * np.maximum(most(u64), most(before)) * per * size / 4 + size * tol / 4
    same_ends(back["grad_gate"][..., gated], gg[..., gated], wide[..., gated], dtype)
    for k in ("out", "h_last", "states"):                # the other channels do not notice
        assert torch.equal(got[k][..., 10:], clean[k][..., 10:])
    for k in back:
        assert torch.equal(back[k][..., 10:], clean_back[k][..., 10:])


@pytest.mark.parametrize("dtype", TYPES)
def test_infinite_states_step_by_step(dtype):
    gate, value = torch.zeros(3, 8, device=DEV, dtype=dtype), torch.ones(3, 8, device=DEV, dtype=dtype)
    gate[1], gate[2] = 3.0, -3.0
    pool = torch.full((3, 8), float("inf"), device=DEV)
    pool[:, 1::2] = -float("inf")
    want = pool.clone()
    for _ in range(3):
        assert torch.equal(api.tac_gated_step(gate, value, pool).float(), want) and torch.equal(pool, want)


@pytest.mark.parametrize("T,B,D,dtype", [(100, 3, 96, torch.float32), (130, 70, 200, torch.bfloat16), (9000, 1, 512, torch.bfloat16)])
def test_infinite_states_where_the_last_takes_the_place_of_the_first(T, B, D, dtype):
    gate, value, lengths, h0, go, gl = (t if t is None else t.contiguous() for t in make(T, B, D, dtype, 34, ragged=B > 1))
    h0[:, ::3], gl[:, 1::3] = float("inf"), -float("inf")
    want = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    want_back = api.tac_gated_scan_backward(gate, value, want["states"], go, lengths=lengths, grad_h_last=gl)
    state, out, states = h0.clone(), torch.empty_like(go), torch.empty_like(want["states"])
    c_abi("tac_gated_scan", T, B, D, dtype, gate, value, lengths, state, out, state, states)
    grad, gg, gv = gl.clone(), torch.empty_like(go), torch.empty_like(go)
    c_abi("tac_gated_scan_backward", T, B, D, dtype, gate, value, lengths, states, go, grad, gg, gv, grad)
    assert torch.isposinf(state[:, ::3]).all() and torch.isneginf(grad[:, 1::3]).all()
    for got, w in ((state, want["h_last"]), (out, want["out"]), (states, want["states"]), (grad, want_back["grad_h0"]), (gg, want_back["grad_gate"]),
                   (gv, want_back["grad_value"])):
        assert torch.allclose(got.float(), w.float(), rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,D", [(50, 2, 66), (3000, 1, 64), (300, 200, 32)])
def test_in_place_a_channel_that_ends_in_nan_keeps_what_was_before(T, B, D, dtype):
    g = torch.Generator(device=DEV).manual_seed(35)
    gate, value, go = ((torch.randn(T, B, D, generator=g, device=DEV) + 1).to(dtype) for _ in range(3))
    clean = api.tac_gated_scan(gate, value, want_states=True)
    clean_back = api.tac_gated_scan_backward(gate, value, clean["states"], go)
    at, nan = T // 2, float("nan")

    def check(got, want, nans):
        """`want`, but NaN in the channels and steps of `nans`"""
        want = want.clone()
        for steps, d in nans:
            want[steps, :, d] = nan
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.5), want.nan_to_num(0.5))
    value[at, :, 3], go[at, :, 5] = nan, nan
    for name in ("value", "gate"):
        a, b = gate.clone(), value.clone()
        into = b if name == "value" else a
        got = api.tac_gated_scan(a, b, out=into, want_states=True)
        check(into, clean["out"], [(slice(at, None), 3)])
        check(got["h_last"][None], clean["h_last"][None], [(slice(None), 3)])
        check(got["states"], clean["states"], [(slice(at // api.TAC_SCAN_CHUNK + 1, None), 3)])
    a, b = gate.clone(), value.clone()
    api.tac_gated_scan_backward(a, b, got["states"], go, grad_gate=a, grad_value=b)
    check(a, clean_back["grad_gate"], [(slice(at, None), 3), (slice(0, at + 1), 5)])
    check(b, clean_back["grad_value"], [(slice(0, at + 1), 5)])
