"""Plain 64-bit implementations of the head norm and of the gated delta rule, step by step from their definitions, for the tests."""
import math

import numpy as np
import torch

from head_util import HALF, U, as64, captured, shifted  # noqa: F401  (the tests' common pieces)

DEV = "cuda:0"


# ---- head norm -----------------------------------------------------------------------------------

def pairs_of(D, sections, interleaved):
    n = sum(sections)
    i = np.arange(n)
    return (2 * i, 2 * i + 1) if interleaved else (i, n + i)


def angles(positions, sections, base):
    p = np.asarray(positions, dtype=np.float64).reshape(len(positions), -1)
    return np.concatenate([p[:, a:a + 1] * np.array([base ** (-i / n) for i in range(n)]) for a, n in enumerate(sections)], 1)


def turned(x, angle, first, second):
    y = x.copy()
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def head_norm(x, gain, eps, positions, sections, base, interleaved):
    rstd = 1.0 if eps is None else 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    y = x * rstd * (1.0 if gain is None else gain)
    return y if positions is None else turned(y, angles(positions, sections, base), *pairs_of(x.shape[-1], sections, interleaved))


def head_norm_backward(x, gain, eps, positions, sections, base, interleaved, grad):
    """(gradient of x, of the gain, the size of the terms that the former is a sum of)"""
    g = grad if positions is None else turned(grad, -angles(positions, sections, base), *pairs_of(x.shape[-1], sections, interleaved))
    rstd = np.ones(x.shape[:-1] + (1,)) if eps is None else 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, w = x * rstd, g * (1.0 if gain is None else gain)
    both = np.abs(n) * np.abs(w * n).mean(-1, keepdims=True)
    grad_x = w if eps is None else rstd * (w - n * (w * n).mean(-1, keepdims=True))
    return grad_x, (g * n).sum((0, 1)), rstd * (np.abs(w) + (0 if eps is None else both))


# ---- gated delta rule ----------------------------------------------------------------------------

def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def delta(q, k, v, gate, write, lengths=None, h0=None):
    """(out, last states, everything that the backward pass wants); float64 arrays [T, B, heads, ..]."""
    T, B, hk, dk = q.shape
    hv, dv = v.shape[2:]
    share = np.arange(hv) // (hv // hk)
    a, b = sigmoid(gate), sigmoid(write)
    S = np.zeros((B, hv, dk, dv)) if h0 is None else h0.copy()
    out, before, us = np.zeros((T, B, hv, dv)), np.zeros((T, B, hv, dk, dv)), np.zeros((T, B, hv, dv))
    for t in range(T):
        before[t] = S
        on = np.ones(B, bool) if lengths is None else t < lengths
        K, Q = k[t][:, share], q[t][:, share]
        faded = a[t][..., None, None] * S
        u = b[t][..., None] * (v[t] - np.einsum("bhkv,bhk->bhv", faded, K))
        new = faded + K[..., None] * u[..., None, :]
        S = np.where(on[:, None, None, None], new, S)
        us[t] = np.where(on[:, None, None], u, 0.0)
        out[t] = np.where(on[:, None, None], np.einsum("bhkv,bhk->bhv", new, Q), 0.0)
    return out, S, (before, us)


def delta_backward(q, k, v, gate, write, kept, grad_out, lengths=None, grad_last=None, chunk=64):
    """Gradients of query, key, value, gate, write and h0, and the size of the terms that a gate's gradient is what is left of where steps are taken a
    chunk at a time: for every step of the chunk from its own on, what queries and keys stand beside, and behind the chunk the state's."""
    T, B, hk, dk = q.shape
    hv, dv = v.shape[2:]
    share = np.arange(hv) // (hv // hk)
    a, b, rest_a, rest_b = sigmoid(gate), sigmoid(write), sigmoid(-gate), sigmoid(-write)
    before, us = kept
    dS = np.zeros((B, hv, dk, dv)) if grad_last is None else grad_last.copy()
    dq, dkey, dvalue, dg, dw = (np.zeros(x.shape) for x in (q, k, v, gate, write))
    sizes, size = np.zeros(gate.shape), np.zeros((B, hv))
    length = lambda x: np.sqrt((x * x).sum(-1))
    for t in range(T - 1, -1, -1):
        on = np.ones(B, bool) if lengths is None else t < lengths
        K, Q = k[t][:, share], q[t][:, share]
        faded = a[t][..., None, None] * before[t]
        after = faded + K[..., None] * us[t][..., None, :]
        D = dS + Q[..., None] * grad_out[t][..., None, :]
        r = np.einsum("bhkv,bhk->bhv", D, K)
        w = b[t][..., None] * r
        live = on[:, None, None]
        one_q = np.where(live, np.einsum("bhkv,bhv->bhk", after, grad_out[t]), 0.0)
        one_k = np.where(live, np.einsum("bhkv,bhv->bhk", D, us[t]) - np.einsum("bhkv,bhv->bhk", faded, w), 0.0)
        for h in range(hv):
            dq[t][:, share[h]] += one_q[:, h]
            dkey[t][:, share[h]] += one_k[:, h]
        dvalue[t] = np.where(live, w, 0.0)
        dw[t] = np.where(live[..., 0], rest_b[t] * (r * us[t]).sum(-1), 0.0)
        if t % chunk == chunk - 1 or t == T - 1:
            size = np.zeros((B, hv))
        last = on & (t == T - 1 if lengths is None else t == np.minimum(lengths, T) - 1) | (t % chunk == chunk - 1)
        size = size + np.where(last[:, None], np.abs(after * dS).sum((-1, -2)), 0.0)
        size = size + length(Q) * length(one_q) + length(r) * length(us[t]) + length(np.einsum("bhkv,bhk->bhv", faded, K)) * length(w)
        sizes[t] = np.where(live[..., 0], rest_a[t] * size, 0.0)
        D = D - K[..., None] * w[..., None, :]
        dg[t] = np.where(live[..., 0], a[t] * rest_a[t] * (D * before[t]).sum((-1, -2)), 0.0)
        dS = np.where(live[..., None], a[t][..., None, None] * D, dS)
    return (dq, dkey, dvalue, dg, dw, dS), sizes


def delta_inputs(T, B, hk, hv, dk, dv, dtype, seed, h0=True, common=1.0, gate=(0.0, 7.0)):
    """Keys of length 1 with a direction in common, values, gates from `gate`, states."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    low, high = gate
    x = dict(query=unit(n(T, B, hk, dk)), key=unit(n(T, B, hk, dk) + common * n(hk, dk)), value=n(T, B, hv, dv),
             gate=n(T, B, hv) + low + (high - low) * torch.rand(hv, generator=g, dtype=torch.float64), write=n(T, B, hv))
    x = {name: t.to(dtype).to(DEV) for name, t in x.items()}
    return x, ((n(B, hv, dk, dv) / math.sqrt(dk)).float().to(DEV) if h0 else None)


def relative(got, want):
    """2-norm of the difference over that of what is wanted."""
    size = float(np.linalg.norm(want))
    off = float(np.linalg.norm(as64(got) - want))
    return off / size if size else off
