"""Angles of far positions against 60 digits, gains' gradients of the longest sums, and heads without keys through the C interface."""
import ctypes
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import delta_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
FAR = [2 ** 31 - 1, -2 ** 31, 10 ** 9, -123456789, 2 ** 24 + 1, 70000, 1, 0]


def exact_turn(position, base, i, n):
    """position base^(-i / n) in turns, less the nearest whole number of them."""
    getcontext().prec = 60
    t = Decimal(position) * (-(Decimal(base).ln()) * i / n).exp() / (2 * PI)
    return float(t - t.to_integral_value())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("base,n", [(10000, 64), (10000, 128), (500000, 64), (100, 7), (1, 3)])
def test_far_positions(base, n, interleaved):
    D, rows = 2 * n, len(FAR)
    x = torch.zeros(rows, 1, D, device=DEV)
    first = slice(0, D, 2) if interleaved else slice(0, n)
    x[..., first] = 1.0
    got = O.as64(api.tac_head_norm(x, positions=torch.tensor(FAR, dtype=torch.int32, device=DEV), base=float(base), interleaved=interleaved)["q"])[:, 0]
    cos, sin = (got[:, 0::2], got[:, 1::2]) if interleaved else (got[:, :n], got[:, n:])
    turn = np.array([[exact_turn(p, base, i, n) for i in range(n)] for p in FAR])
    # The frequency: log2(base) and its part of n (a rounding each) times i, of which an error of e is ln 2 e in 2^-x; 2^-x itself (2), 1 / 2 pi, their product and that
    # with the position (half each, and what is left of the product's two).  Then the fraction of a turn in float32, less than 2^-26 of a whole one, sine and cosine (2), and two
    # products' roundings
    part = np.log2(base) * np.arange(n) / n
    angle = np.abs(np.array(FAR, dtype=np.float64))[:, None] * base ** (-np.arange(n) / n)
    bound = angle * (np.log(2) * 3 * part + 4) * 2.0 ** -53 + 2 * np.pi * 2.0 ** -26 + 4 * O.U
    for name, mine, want in (("cos", cos, np.cos(2 * np.pi * turn)), ("sin", sin, np.sin(2 * np.pi * turn))):
        off = np.abs(mine - want)
        assert (off <= bound).all(), (name, float((off / bound).max()))


@pytest.mark.parametrize("rows,hq,hk,D", [(12000, 1, 1, 512), (7000, 3, 1, 256), (30000, 2, 1, 64)])
def test_gradients_of_gains_over_many_rows(rows, hq, hk, D):
    g = torch.Generator(device=DEV).manual_seed(D)
    q, k = (torch.randn(rows, h, D, generator=g, device=DEV) for h in (hq, hk))
    dq, dk = (torch.randn(rows, h, D, generator=g, device=DEV) for h in (hq, hk))
    back = api.tac_head_norm_backward(q, k, None, None, dq, dk, eps=1e-6)
    lanes = 64 if D > 256 else 32 if D > 128 else 16 if D > 64 else 8
    # at most 768 workgroups of 256 / lanes groups: of each the heads one after the other; over a workgroup's groups; 768 rows in 16 slices, and those.  A term is a
    # statistic (a sum of up to 8 in a lane and 6 joinings, half of it in the root; a root and a division, 2 each) and three products
    terms = -(-rows * (hq + hk) // (768 * (256 // lanes))) + 256 // lanes + 48 + 16 + 7 + 4 + 3
    for name, x, d in (("grad_gain_q", q, dq), ("grad_gain_k", k, dk)):
        x64, d64 = x.double(), d.double()
        one = d64 * x64 / torch.sqrt(x64.square().mean(-1, keepdim=True) + 1e-6)
        want, size = one.sum((0, 1)).cpu().numpy(), one.abs().sum((0, 1)).cpu().numpy()
        assert (np.abs(O.as64(back[name]) - want) <= terms * O.U * size).all(), name


def test_without_keys_through_the_c_interface():
    """Whatever stands for the keys, queries' own tensors for instance, is neither read nor written."""
    g = torch.Generator(device=DEV).manual_seed(3)
    q, dq, gain = torch.randn(9, 3, 32, generator=g, device=DEV), torch.randn(9, 3, 32, generator=g, device=DEV), torch.ones(32, device=DEV)
    want, back = api.tac_head_norm(q, None, gain, eps=1e-6)["q"], api.tac_head_norm_backward(q, None, gain, None, dq, eps=1e-6)
    s = api.tac_head_strides_t
    d = api.tac_head_norm_desc_t(rows=9, query_heads=3, key_heads=0, D=32, dtype=api.TAC_FP32, axes=0, eps=1e-6, **{n: s(96, 32) for n in ("query", "out_query", "grad_query")},
                                 **{n: s(-5, 0) for n in ("key", "out_key", "grad_key")})
    out, grad, sums = torch.empty_like(q), torch.empty_like(q), torch.empty(32, device=DEV)
    work = torch.empty(api.lib().tac_head_norm_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device=DEV)
    p, stream = lambda t: t.data_ptr(), torch.cuda.current_stream().cuda_stream
    assert api.lib().tac_head_norm(ctypes.byref(d), p(q), p(out), p(gain), p(out), None, p(out), p(out), stream) == 0
    assert api.lib().tac_head_norm_backward(ctypes.byref(d), p(q), p(q), p(gain), p(grad), None, p(dq), p(dq), p(grad), p(q), p(sums), p(sums), p(work), stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(grad, back["grad_q"]) and torch.equal(sums, back["grad_gain_q"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [16, 512])
def test_large_magnitudes(D, dtype):
    """A head's squares are summed in float32: up to 2^59 they have room, whatever the head's size; where they have not, the results are zero."""
    x = torch.full((2, 1, D), 2.0 ** 59, device=DEV, dtype=dtype)
    x[..., ::2] *= -1
    x[1] *= 2.0 ** 6
    got = api.tac_head_norm(x, eps=1e-6)["q"].float()
    # 8 terms in a lane and 6 joinings, half of it in the root; a root and a division (2 each), a product; the result's own rounding
    assert ((got[0] - torch.sign(x[0].float())).abs() <= (7 + 4 + 1) * O.U + O.HALF[dtype]).all()
    assert (got[1] == 0).all()
