"""Norm of heads with the rotation by position, and its backward pass, against 64 bits."""
import numpy as np
import pytest
import torch

import delta_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
TYPES = [torch.float32, torch.bfloat16]
# y from float32: the sum of squares has 8 terms in a lane and 6 joinings, half of whose error reaches rstd; 1/sqrt and division (2 each), two products,
# sine and cosine (an angle of 64 bits rounded to half a turn's 2^-24, pi of it; 2 of the functions), one product and one sum: relative to a pair's size
Y32 = (7 + 4 + 2 + 4 + 2 + 2) * O.U


def make(rows, hq, hk, D, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    both = (n(rows, (hq + hk) * D) * torch.exp(n((hq + hk) * D))).to(dtype)
    q, k = both[:, :hq * D].view(rows, hq, D), both[:, hq * D:].view(rows, hk, D)
    return q, k if hk else None, 1 + 0.3 * n(D), 1 + 0.3 * n(D) if hk else None, n(rows, hq, D).to(dtype), n(rows, hk, D).to(dtype) if hk else None


def positions_of(rows, axes, far, seed=3):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-far, far + 1, (rows, axes), generator=g, dtype=torch.int32)
    p[0] = 0
    return (p[:, 0].contiguous() if axes == 1 else p).to(DEV)


def pair_size(y, sections, interleaved):
    """A feature's size, or that of its pair where it is turned."""
    size = np.abs(y)
    if sections:
        f, s = O.pairs_of(y.shape[-1], sections, interleaved)
        both = np.hypot(y[..., f], y[..., s])
        size[..., f], size[..., s] = both, both
    return size


def check(q, k, gq, gk, how, sections):
    """Forward and backward against 64 bits; returns the results."""
    rows, hq, D = q.shape
    half = O.HALF[q.dtype]
    positions = None if how.get("positions") is None else how["positions"].cpu().numpy()
    args = (how.get("eps"), positions, sections, how.get("base", 10000.0), how.get("interleaved", False))
    got = api.tac_head_norm(q, k, gq, gk, **how)
    g = torch.Generator(device=DEV).manual_seed(9)
    grads = [None if x is None else torch.randn(x.shape, generator=g, device=DEV).to(x.dtype) for x in (q, k)]
    back = api.tac_head_norm_backward(q, k, gq, gk, *grads, **how)
    for name, x, gain, grad in (("q", q, gq, grads[0]), ("k", k, gk, grads[1])):
        if x is None:
            assert got["k"] is None and back["grad_k"] is None and back["grad_gain_k"] is None
            continue
        x64, gain64, grad64 = O.as64(x), None if gain is None else O.as64(gain), O.as64(grad)
        y = O.head_norm(x64, gain64, *args)
        assert (np.abs(O.as64(got[name]) - y) <= half * (1 + 1e-6) * np.abs(y) + Y32 * pair_size(y, sections, args[4])).all(), name
        gx, gg, size = O.head_norm_backward(x64, gain64, *args, grad64)
        # terms of a pair that is turned have the pair's size; the mean is a sum as above
        size = pair_size(size, sections, args[4]) + np.abs(gx)
        assert (np.abs(O.as64(back["grad_" + name]) - gx) <= half * (1 + 1e-6) * np.abs(gx) + 3 * Y32 * size).all(), name
        # a lane's heads one after the other (rows and heads over 1024 workgroups of 4 or more), up to 32 lanes of a workgroup, 64 workgroups, 16 slices
        terms = rows * (hq + (0 if k is None else k.shape[1])) / 4096 + 4 + 32 + 64 + 16
        sizes = (pair_size(grad64, sections, args[4]) * np.abs(x64 * (1 if args[0] is None else 1 / np.sqrt((x64 ** 2).mean(-1, keepdims=True) + args[0])))).sum((0, 1))
        assert (np.abs(O.as64(back["grad_gain_" + name]) - gg) <= (terms + Y32 / O.U) * O.U * sizes).all(), name
    return got, back


SHAPES = [  # rows, query heads, key heads, features, sections
    (1, 1, 1, 2, (1,)), (1, 1, 0, 16, (8,)), (3, 2, 1, 10, (2, 1)), (5, 4, 2, 64, (32,)), (4, 3, 3, 66, (33,)), (7, 16, 8, 128, (64,)), (6, 4, 1, 128, (16,)),
    (2, 2, 2, 96, (8, 20, 20)), (9, 8, 2, 256, (128,)), (2, 1, 1, 250, (3, 4, 5, 6)), (3, 2, 2, 512, (100, 156)), (2, 1, 3, 514 - 2, (1,)), (33, 5, 3, 40, (7, 5, 8))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk,D,sections", SHAPES)
def test_forward_and_backward(rows, hq, hk, D, sections, interleaved, dtype):
    q, k, gq, gk, _, _ = make(rows, hq, hk, D, dtype, 100 + D)
    check(q, k, gq, gk, dict(eps=EPS, positions=positions_of(rows, len(sections), 300), sections=sections, interleaved=interleaved), sections)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,hq,hk,D", [(700, 16, 8, 128), (5000, 2, 1, 64), (40000, 1, 1, 16), (300, 64, 8, 32)])
def test_more_heads_than_a_launch_takes_at_once(rows, hq, hk, D, dtype):
    q, k, gq, gk, _, _ = make(rows, hq, hk, D, dtype, 7)
    how = dict(eps=EPS, positions=positions_of(rows, 1, 10000))
    got, back = check(q, k, gq, gk, how, (D // 2,))
    again = api.tac_head_norm_backward(q, k, gq, gk, got["q"], got["k"], **how)
    once_more = api.tac_head_norm_backward(q, k, gq, gk, got["q"], got["k"], **how)
    assert all(torch.equal(again[n], once_more[n]) for n in again)              # no order of arrival


@pytest.mark.parametrize("dtype", TYPES)
def test_far_positions_have_the_precision_of_near_ones(dtype):
    rows = 64
    q, k, gq, gk, _, _ = make(rows, 2, 1, 128, dtype, 8)
    p = torch.tensor([2 ** 31 - 1, -2 ** 31, 10 ** 9, 123456789] * 16, dtype=torch.int32, device=DEV)
    check(q, k, gq, gk, dict(eps=EPS, positions=p), (64,))
    check(q, k, gq, gk, dict(eps=EPS, positions=p, base=500000.0), (64,))


@pytest.mark.parametrize("dtype", TYPES)
def test_without_norm_rotation_gain_or_keys(dtype):
    q, k, gq, gk, _, _ = make(19, 4, 2, 48, dtype, 9)
    p = positions_of(19, 1, 50)
    check(q, k, gq, gk, dict(eps=EPS), ())
    check(q, k, None, None, dict(eps=EPS, positions=p), (24,))
    check(q, k, None, gk, dict(positions=p), (24,))
    check(q, None, gq, None, dict(eps=EPS, positions=p, sections=(5,)), (5,))
    back = api.tac_head_norm_backward(q, k, gq, gk, q, k, eps=EPS, want_grad_gain=False)
    assert back["grad_gain_q"] is None and back["grad_gain_k"] is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,sections", [(4, (1,)), (8, (3,)), (10, (5,)), (18, (2, 3)), (70, (9,)), (254, (31, 1, 70)), (512, (254, 1))])
def test_heads_that_are_no_whole_pieces(D, sections, interleaved, dtype):
    """Odd numbers of pairs, rows at any address with NaN between them: the same values as from whole rows, and nothing beside the results is written."""
    rows, hq, hk = 9, 3, 1
    q, k, gq, gk, dq, dk = make(rows, hq, hk, D, dtype, 20 + D)
    how = dict(eps=EPS, positions=positions_of(rows, len(sections), 200), sections=sections, interleaved=interleaved)
    plain, _ = check(q, k, gq, gk, how, sections)
    back = api.tac_head_norm_backward(q.contiguous(), k.contiguous(), gq, gk, dq, dk, **how)
    pad = lambda t, by=3: torch.nn.functional.pad(t, (1, by), value=float("nan"))
    inner = lambda t: t[..., 1:1 + D]
    room = {n: torch.full((rows, h, D + 4), 7.0, dtype=dtype, device=DEV) for n, h in (("q", hq), ("k", hk))}
    got = api.tac_head_norm(inner(pad(q)), inner(pad(k)), gq, gk, out_query=inner(room["q"]), out_key=inner(room["k"]), **how)
    for n in got:
        assert torch.equal(got[n], plain[n])
        assert (room[n][..., 0] == 7).all() and (room[n][..., 1 + D:] == 7).all()
    again = api.tac_head_norm_backward(inner(pad(q)), inner(pad(k)), gq, gk, inner(pad(dq)), inner(pad(dk)), grad_query=inner(room["q"]), grad_key=inner(room["k"]), **how)
    assert all(torch.equal(again[n], back[n]) for n in back)
    assert all((t[..., 0] == 7).all() and (t[..., 1 + D:] == 7).all() for t in room.values())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_addresses_and_in_place(interleaved, dtype):
    rows, hq, hk, D = 21, 3, 2, 64
    q, k, gq, gk, dq, dk = make(rows, hq, hk, D, dtype, 10)
    how = dict(eps=EPS, positions=positions_of(rows, 1, 99), interleaved=interleaved)
    plain = api.tac_head_norm(q.contiguous(), k.contiguous(), gq, gk, **how)
    back = api.tac_head_norm_backward(q.contiguous(), k.contiguous(), gq, gk, dq, dk, **how)
    for f in (lambda t: t, O.shifted, lambda t: torch.stack([t, torch.full_like(t, float("nan"))], 2).flatten(1, 2)[:, ::2], lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)):
        room = {n: f(torch.zeros_like(t.contiguous())) for n, t in (("q", q), ("k", k))}
        got = api.tac_head_norm(f(q), f(k), gq, gk, out_query=room["q"], out_key=room["k"], **how)
        assert got["q"] is room["q"] and torch.equal(got["q"], plain["q"]) and torch.equal(got["k"], plain["k"])
        again = api.tac_head_norm_backward(f(q), f(k), gq, gk, f(dq), f(dk), grad_query=room["q"], grad_key=room["k"], **how)
        assert all(torch.equal(again[n], back[n]) for n in back)
    x, y = q.contiguous().clone(), k.contiguous().clone()
    api.tac_head_norm(x, y, gq, gk, out_query=x, out_key=y, **how)
    assert torch.equal(x, plain["q"]) and torch.equal(y, plain["k"])
    x, y = dq.clone(), dk.clone()
    api.tac_head_norm_backward(q, k, gq, gk, x, y, grad_query=x, grad_key=y, **how)
    assert torch.equal(x, back["grad_q"]) and torch.equal(y, back["grad_k"])


def test_gradient_against_differences_of_the_kernel():
    q, k, gq, gk, dq, dk = make(6, 3, 2, 32, torch.float32, 12)
    how = dict(eps=EPS, positions=positions_of(6, 1, 40))
    back = api.tac_head_norm_backward(q, k, gq, gk, dq, dk, **how)
    loss = lambda q, k, gq, gk: float(sum((r.double() * d.double()).sum() for r, d in zip(api.tac_head_norm(q, k, gq, gk, **how).values(), (dq, dk))))
    g = torch.Generator(device=DEV).manual_seed(13)
    for i, name in enumerate(("grad_q", "grad_k", "grad_gain_q", "grad_gain_k")):
        given = [q, k, gq, gk]
        way = torch.randn(given[i].shape, generator=g, device=DEV)
        h = 2.0 ** -7
        ends = []
        for s in (h, -h):
            moved = list(given)
            moved[i] = given[i] + s * way
            ends.append(loss(*moved))
        want = float((back[name].double() * way.double()).sum())
        # the difference's own curvature (h^2 times the third derivative, of the size of the terms) and the results' rounding over 2 h
        size = float((back[name].double().abs() * way.double().abs()).sum())
        assert abs((ends[0] - ends[1]) / (2 * h) - want) <= 20 * h * h * size + 1e-4 * size, name


def test_nan_stays_in_its_head_and_rows_of_zeros():
    q, k, gq, gk, dq, dk = make(8, 3, 2, 64, torch.float32, 14)
    q, k = q.contiguous(), k.contiguous()
    how = dict(eps=EPS, positions=positions_of(8, 1, 40))
    plain = api.tac_head_norm(q, k, gq, gk, **how)
    q[2, 1, 5], k[7, 0, 63] = float("nan"), float("inf")
    q[4] = 0
    got = api.tac_head_norm(q, k, gq, gk, **how)
    assert torch.isnan(got["q"][2, 1]).all() and (got["q"][4] == 0).all()
    same = torch.ones(8, 3, dtype=torch.bool, device=DEV)
    same[2, 1], same[4] = False, False
    assert torch.equal(got["q"][same], plain["q"][same])
    same = torch.ones(8, 2, dtype=torch.bool, device=DEV)
    same[7, 0] = False
    assert torch.equal(got["k"][same], plain["k"][same])


def test_captured_and_replayed():
    q, k, gq, gk, dq, dk = make(100, 4, 2, 128, torch.bfloat16, 15)
    how = dict(eps=EPS, positions=positions_of(100, 1, 4000))

    def call():
        r = api.tac_head_norm(q, k, gq, gk, **how)
        r.update(api.tac_head_norm_backward(q, k, gq, gk, dq, dk, **how))
        return r
    want = {n: t.clone() for n, t in call().items()}
    for r in O.captured(call):
        assert all(torch.equal(r[n], want[n]) for n in want)
        for t in r.values():
            t.zero_()
