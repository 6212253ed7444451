"""Plain 64-bit implementations of the dense operators, written from their definitions, for the tests."""
import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # half a step relative to the value
U = 2.0 ** -24                                                       # one rounding to float32


def block_exponents(v, block=128):
    """Per row and block of columns, the smallest e >= -127 with max |finite| <= 448 * 2^e.  v: float64 array [R, C]."""
    R, C = v.shape
    kb = -(-C // block)
    w = np.zeros((R, kb * block))
    w[:, :C] = np.where(np.isfinite(v), np.abs(v), 0.0)
    top = w.reshape(R, kb, block).max(2)
    e = np.full(top.shape, -127, dtype=np.int64)
    some = top > 448 * 2.0 ** -127
    e[some] = np.ceil(np.log2(top[some] / 448.0)).astype(np.int64)
    for _ in range(2):                                                # log2 may be off at exact powers of two
        e = np.where(top > 448 * np.exp2(e.astype(float)), e + 1, e)
        e = np.where((top <= 448 * np.exp2(e - 1.0)) & (e > -127), e - 1, e)
    return e


def e4m3(r):
    """Nearest (even) e4m3 number of |r| <= 448, subnormals included; NaN where r is not finite."""
    r = np.asarray(r, dtype=np.float64)
    ok = np.isfinite(r)
    s = np.where(ok, r, 0.0)
    x = np.maximum(np.frexp(s)[1] - 1, -6)
    step = np.exp2(x - 3.0)
    return np.where(ok, np.round(s / step) * step, np.nan)            # np.round: half to even


def quantized(v, tiles=False):
    """(values, exponents per row and block) of a float64 matrix in 8 bits along its rows."""
    R, C = v.shape
    e = block_exponents(v)
    if tiles:
        for r in range(0, R, 128):
            e[r:r + 128] = e[r:r + 128].max(0)
    unit = np.exp2(np.repeat(e, 128, axis=1)[:, :C].astype(float))
    return e4m3(v / unit) * unit, e


def decode(matrix, cols):
    """The float64 values of an 8-bit matrix (codes, scales), bit by bit, and its exponents."""
    codes, scales = matrix[0].cpu().numpy().astype(np.int64), matrix[1].cpu().numpy().astype(np.int64)
    R, kb = codes.shape[0], codes.shape[1] // 128
    x, f = (codes >> 3) & 15, (codes & 7).astype(float)
    v = np.where(x == 0, f * 2.0 ** -9, (8 + f) * np.exp2(x - 10.0))
    v = np.where((codes & 127) == 127, np.nan, v) * np.where(codes >= 128, -1.0, 1.0)
    e = scales[:, :kb] - 127
    return (v * np.exp2(np.repeat(e, 128, axis=1).astype(float)))[:, :cols], e


def pads_are_zero(matrix, cols):
    codes, scales = matrix
    kb = codes.shape[1] // 128
    return int(codes[:, cols:].sum()) == 0 and int(scales[:, kb:].sum()) == 0


def norm(x, residual, gain, eps):
    s = x if residual is None else x + residual
    rstd = 1.0 / np.sqrt((s * s).mean(1) + eps)
    return s, rstd, s * rstd[:, None] * (1.0 if gain is None else gain)


def norm_backward(h, rstd, gain, gy, gh):
    n = h * rstd[:, None]
    w = gy * (1.0 if gain is None else gain)
    gx = rstd[:, None] * (w - n * (w * n).mean(1, keepdims=True))
    return gx + (0.0 if gh is None else gh), (gy * n).sum(0)


def scan(gate, value, lengths=None, h0=None):
    """(out, states before every step, last states), float64 [T, B, D]."""
    T, B, D = gate.shape
    with np.errstate(over="ignore"):
        a, rest = 1.0 / (1.0 + np.exp(-gate)), 1.0 / (1.0 + np.exp(gate))
    h = np.zeros((B, D)) if h0 is None else h0.copy()
    out, before = np.zeros((T, B, D)), np.zeros((T, B, D))
    for t in range(T):
        before[t] = h
        on = np.ones((B, 1), bool) if lengths is None else (t < lengths)[:, None]
        h = np.where(on, a[t] * h + rest[t] * value[t], h)
        out[t] = np.where(on, h, 0.0)
    return out, before, h


def scan_backward(gate, value, before, grad_out, lengths=None, grad_last=None):
    T, B, D = gate.shape
    with np.errstate(over="ignore"):
        a, rest = 1.0 / (1.0 + np.exp(-gate)), 1.0 / (1.0 + np.exp(gate))
    c = np.zeros((B, D)) if grad_last is None else grad_last.copy()
    gg, gv = np.zeros((T, B, D)), np.zeros((T, B, D))
    for t in range(T - 1, -1, -1):
        on = np.ones((B, 1), bool) if lengths is None else (t < lengths)[:, None]
        here = c + grad_out[t]
        gv[t] = np.where(on, rest[t] * here, 0.0)
        gg[t] = np.where(on, here * (before[t] - value[t]) * a[t] * rest[t], 0.0)
        c = np.where(on, a[t] * here, c)
    return gg, gv, c


def as64(t):
    return t.detach().cpu().double().numpy()


def strided(t, extra):
    """The same matrix (or sequence) inside a wider one: rows further apart than they are long."""
    room = torch.full(t.shape[:-1] + (t.shape[-1] + extra,), float("nan"), dtype=t.dtype, device=t.device)
    room[..., :t.shape[-1]] = t
    return room[..., :t.shape[-1]]


def shifted(t):
    """The same matrix from an address that is one element off."""
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    v = room[1:].view(t.shape)
    v.copy_(t)
    return v


def captured(call, replays=3):
    """Runs `call` under a graph capture after one eager run; yields after every replay."""
    call()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        result = call()
    for _ in range(replays):
        graph.replay()
        torch.cuda.synchronize()
        yield result
