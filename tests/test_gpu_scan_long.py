"""The gated recurrence and its backward pass over hundreds and thousands of steps against 64 bits, with a bound of its own for every step and channel."""
import numpy as np
import pytest
import torch

import head_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# sequences in parts of one tile (128 steps), in parts of several, and whole (from 192 groups of 64 or 128 channels on); odd channels
SHAPES = [(511, 1, 48), (512, 2, 64), (1030, 1, 200), (2500, 3, 41), (5000, 1, 17), (9000, 1, 512), (3000, 60, 64), (400, 200, 66), (1500, 64, 30)]


def bounds(g, u, h0, go, gl, lengths):
    """The results in 64 bits and how far float32 may be off, step by step.  To first order in U = 2^-24:

    w = min(a, 1 - a) = exp(-|g|) / (1 + exp(-|g|)) is off by (2 |g| + 8) U of itself (the exponent's argument and its constant, exp, sum, 1 / x, product).
    A step h + w (u - h) (or u - w (u - h)) rounds its result once and the difference once and carries w's error; a join of maps over 16 steps rounds
    once more.  With H the recurrence of the magnitudes |h0|, |u| (the maps start from 0, so |h| itself does not bound what they round),
        e_t = a_t e_{t-1} + U (1.5 H_t + (2 |g_t| + 10) w_t (|u_t| + H_{t-1})),
    and the same backwards for the gradient n_t = c_t that arrives at step t's state, with C the recurrence of the magnitudes of its sources."""
    T, B, D = g.shape
    with np.errstate(over="ignore"):
        a, rest = 1.0 / (1.0 + np.exp(-g)), 1.0 / (1.0 + np.exp(g))
    w, off = np.minimum(a, rest), (2 * np.abs(g) + 10) * O.U
    on = np.ones((T, B, 1), bool) if lengths is None else (np.arange(T)[:, None] < lengths[None, :])[..., None]
    r = {k: np.zeros((T, B, D)) for k in ("out", "before", "e_out", "e_before", "gg", "gv", "e_gg", "e_gv")}
    h, H, e = h0.copy(), np.abs(h0), np.zeros((B, D))
    mags = np.zeros((T, B, D))
    for t in range(T):
        r["before"][t], r["e_before"][t], mags[t] = h, e, H
        H1 = a[t] * H + rest[t] * np.abs(u[t])
        e = np.where(on[t], a[t] * e + 1.5 * O.U * H1 + off[t] * w[t] * (np.abs(u[t]) + H), e)
        h, H = np.where(on[t], a[t] * h + rest[t] * u[t], h), np.where(on[t], H1, H)
        r["out"][t], r["e_out"][t] = np.where(on[t], h, 0.0), np.where(on[t], e, 0.0)
    r["h_last"], r["e_h_last"] = h, e
    c, C, e = gl.copy(), np.abs(gl), np.zeros((B, D))
    for t in range(T - 1, -1, -1):
        now, N = c + go[t], C + np.abs(go[t])
        e_now = e + O.U * N
        diff, size = r["before"][t] - u[t], mags[t] + np.abs(u[t])
        r["gv"][t], r["e_gv"][t] = np.where(on[t], rest[t] * now, 0.0), np.where(on[t], rest[t] * (e_now + off[t] * N), 0.0)
        r["gg"][t] = np.where(on[t], now * a[t] * rest[t] * diff, 0.0)
        r["e_gg"][t] = np.where(on[t], a[t] * rest[t] * (e_now * size + N * (r["e_before"][t] + (off[t] + 4 * O.U) * size)), 0.0)
        e = np.where(on[t], a[t] * e_now + 1.5 * O.U * a[t] * N + off[t] * w[t] * N, e)
        c, C = np.where(on[t], a[t] * now, c), np.where(on[t], a[t] * N, C)
    r["g0"], r["e_g0"] = c, e
    return r


def close(got, r, name, error, dtype):
    want, tol = r[name], 1.01 * r[error]
    # a bound that could not tell a result from zeros would hold nothing
    rms = np.sqrt((want ** 2).mean())
    assert np.sqrt((tol ** 2).mean()) < 2 ** -6 * rms, (name, np.sqrt((tol ** 2).mean()), rms)
    half = O.HALF[dtype]
    off = np.abs(O.as64(got) - want)
    assert (off <= half * (np.abs(want) + tol) * (1 + 1e-6) + tol + 1e-37).all(), (name, (off / (half * np.abs(want) + tol + 1e-37)).max())


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,D", SHAPES)
def test_every_step_within_its_own_bound(T, B, D, dtype, ragged):
    g = torch.Generator(device=DEV).manual_seed(900 + T)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    both = n(T, B, 2 * D)
    both[..., :D] += 6 * torch.rand(D, generator=g, device=DEV)          # channels that forget within a few steps to some hundreds
    both, h0, go, gl = both.to(dtype), n(B, D), n(T, B, D).to(dtype), n(B, D)
    gate, value, lengths = both[..., :D], both[..., D:], None
    if ragged:
        lengths = torch.randint(T // 2, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        if B > 1:
            lengths[0], lengths[1] = 0, T
    r = bounds(*(O.as64(t) for t in (gate, value, h0, go, gl)), None if lengths is None else lengths.cpu().numpy())
    got = api.tac_gated_scan(gate, value, lengths=lengths, h0=h0, want_states=True)
    close(got["out"], r, "out", "e_out", dtype)
    close(got["h_last"], r, "h_last", "e_h_last", torch.float32)
    r["states"], r["e_states"] = r["before"][::api.TAC_SCAN_CHUNK], r["e_before"][::api.TAC_SCAN_CHUNK]
    close(got["states"], r, "states", "e_states", torch.float32)
    back = api.tac_gated_scan_backward(gate, value, got["states"], go, lengths=lengths, grad_h_last=gl)
    close(back["grad_value"], r, "gv", "e_gv", dtype)
    close(back["grad_gate"], r, "gg", "e_gg", dtype)
    close(back["grad_h0"], r, "g0", "e_g0", torch.float32)
