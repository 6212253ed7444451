"""Residual norm and its backward pass against 64 bits."""
import numpy as np
import pytest
import torch

import head_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
TYPES = [torch.float32, torch.bfloat16]
# y from float32: one rounding of the sum, two products, 1/sqrt and division (2 each), and the sum of squares: at most 32 terms in a lane
# and ten halvings of lanes and waves, half of whose relative error reaches rstd
Y32 = (3 + 4 + 21) * O.U


def make(rows, cols, dtype, seed, residual=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    spread = torch.exp(n(cols))
    x, r = (n(rows, cols) * spread).to(dtype), (2 * n(rows, cols)).to(dtype) if residual else None
    return x, r, 1 + 0.3 * n(cols), (n(rows, cols)).to(dtype), n(rows, cols).to(dtype)


def check_forward(x, r, gain, got):
    half = O.HALF[x.dtype]
    s, rstd, y = O.norm(O.as64(x), None if r is None else O.as64(r), None if gain is None else O.as64(gain), EPS)
    if got["h"] is not None:
        assert (np.abs(O.as64(got["h"]) - s) <= half * (1 + 1e-6) * np.abs(s) + O.U * np.abs(s)).all()
    if got["rstd"] is not None:
        assert (np.abs(O.as64(got["rstd"]) - rstd) <= Y32 * rstd).all()
    if got["y"] is not None:
        assert (np.abs(O.as64(got["y"]) - y) <= (half + Y32) * (1 + 1e-6) * np.abs(y)).all()
    if got["scaled"] is not None:
        cols = x.shape[1]
        v, e = O.decode(got["scaled"], cols)
        low, high = O.block_exponents(y * (1 - 2 * Y32)), O.block_exponents(y * (1 + 2 * Y32))
        assert ((e == low) | (e == high)).all() and O.pads_are_zero(got["scaled"], cols)
        unit = np.exp2(np.repeat(e, 128, axis=1).astype(float))[:, :cols]
        assert (np.abs(v - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * unit) + Y32 * np.abs(y)).all()
    return s, rstd


def check_backward(h, rstd64, gain, gy, gh, got):
    half = O.HALF[h.dtype]
    rows, cols = h.shape
    h64, gy64 = O.as64(h), O.as64(gy)
    g64 = 1.0 if gain is None else O.as64(gain)
    gx, gg = O.norm_backward(h64, rstd64, None if gain is None else g64, gy64, None if gh is None else O.as64(gh))
    # every term's own size: |w|, |n| mean|w n| (a sum of `cols` terms, as above) and |grad_h|
    n, w = h64 * rstd64[:, None], gy64 * g64
    size = rstd64[:, None] * (np.abs(w) + np.abs(n) * np.abs(w * n).mean(1, keepdims=True)) + (0 if gh is None else np.abs(O.as64(gh)))
    assert (np.abs(O.as64(got["grad_x"]) - gx) <= (half * np.abs(gx) + 3 * Y32 * size) * (1 + 1e-6)).all()
    if got["grad_gain"] is not None:
        # rows of a workgroup one after the other, then up to 64 partial sums in a row and 16 of those
        terms = rows / 1024 + 4 + 80
        assert (np.abs(O.as64(got["grad_gain"]) - gg) <= (terms + Y32 / O.U) * O.U * np.abs(gy64 * n).sum(0)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (5, 8), (3, 127), (4, 128), (9, 129), (2, 512), (7, 520), (6, 1000), (5, 1024), (3, 1025),
                                       (33, 2048), (2, 3001), (17, 4096), (2, 4104), (3, 8192), (2, 9000), (2, 16384), (2, 20000), (1, 32768)])
def test_forward_and_backward(rows, cols, dtype):
    x, r, gain, gy, gh = make(rows, cols, dtype, 100 + cols)
    got = api.tac_residual_norm(x, r, gain, eps=EPS, want_scaled=True, want_rstd=True)
    _, rstd64 = check_forward(x, r, gain, got)
    check_backward(got["h"], rstd64, gain, gy, gh, api.tac_residual_norm_backward(got["h"], gain, got["rstd"], gy, gh))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1500, 264), (5000, 64), (2100, 1536)])
def test_more_rows_than_workgroups(rows, cols, dtype):
    x, r, gain, gy, gh = make(rows, cols, dtype, 7)
    got = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True)
    _, rstd64 = check_forward(x, r, gain, got)
    back = api.tac_residual_norm_backward(got["h"], gain, got["rstd"], gy, gh)
    check_backward(got["h"], rstd64, gain, gy, gh, back)
    again = api.tac_residual_norm_backward(got["h"], gain, got["rstd"], gy, gh)
    assert torch.equal(back["grad_gain"], again["grad_gain"])          # no order of arrival


@pytest.mark.parametrize("dtype", TYPES)
def test_without_residual_gain_and_gradient_past_the_norm(dtype):
    x, _, _, gy, _ = make(19, 300, dtype, 8, residual=False)
    got = api.tac_residual_norm(x, eps=EPS, want_rstd=True, want_scaled=True)
    assert got["h"] is None
    _, rstd64 = check_forward(x, None, None, got)
    check_backward(x, rstd64, None, gy, None, api.tac_residual_norm_backward(x, None, got["rstd"], gy))
    only = api.tac_residual_norm_backward(x, None, got["rstd"], gy, want_grad_gain=False)
    assert only["grad_gain"] is None
    check_backward(x, rstd64, None, gy, None, only)
    for want in (dict(want_y=False, want_scaled=True), dict(want_y=False, want_h=True), dict(want_y=False, want_rstd=True)):
        check_forward(x, None, None, api.tac_residual_norm(x, eps=EPS, **want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [96, 1000, 2048])
@pytest.mark.parametrize("move", ["strided", "shifted"])
def test_strides_and_addresses(cols, dtype, move):
    x, r, gain, gy, gh = make(11, cols, dtype, 9)
    plain = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True, want_scaled=True)
    back = api.tac_residual_norm_backward(plain["h"], gain, plain["rstd"], gy, gh)
    f = (lambda t: O.strided(t, 5)) if move == "strided" else O.shifted
    g = gain if move == "strided" else O.shifted(gain)
    moved = api.tac_residual_norm(f(x), f(r), g, eps=EPS, want_rstd=True, want_scaled=True)
    for k in ("h", "y", "rstd"):
        assert torch.equal(moved[k], plain[k]), k
    assert torch.equal(moved["scaled"][0], plain["scaled"][0]) and torch.equal(moved["scaled"][1], plain["scaled"][1])
    out = f(torch.zeros_like(x))
    again = api.tac_residual_norm_backward(f(plain["h"]), g, plain["rstd"], f(gy), f(gh), grad_x=out)
    assert torch.equal(out, back["grad_x"]) and torch.equal(again["grad_gain"], back["grad_gain"])
    if move == "strided":                                        # what stands between the rows is left alone
        room = out.as_strided((11, cols + 5), (cols + 5, 1))
        assert torch.isnan(room[:, cols:]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(dtype):
    x, r, gain, gy, gh = make(40, 1200, dtype, 10)
    plain = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True)
    back = api.tac_residual_norm_backward(plain["h"], gain, plain["rstd"], gy, gh)
    stream = r.clone()
    got = api.tac_residual_norm(x, stream, gain, eps=EPS, h=stream)
    assert torch.equal(stream, plain["h"]) and torch.equal(got["y"], plain["y"])
    for name in ("gy", "gh"):
        a, b = gy.clone(), gh.clone()
        into = a if name == "gy" else b
        api.tac_residual_norm_backward(plain["h"], gain, plain["rstd"], a, b, grad_x=into)
        assert torch.equal(into, back["grad_x"])


def test_rows_of_zeros_infinities_and_nan():
    x, _, gain, _, _ = make(6, 400, torch.float32, 11, residual=False)
    x[1] = 0
    x[2, 5], x[3, 399] = float("inf"), float("nan")
    got = api.tac_residual_norm(x, None, gain, eps=EPS, want_scaled=True, want_rstd=True)
    keep = [0, 1, 4, 5]
    check_forward(x[keep], None, gain, dict(h=None, y=got["y"][keep], rstd=got["rstd"][keep],
                                            scaled=(got["scaled"][0][keep], got["scaled"][1][keep])))
    assert (got["y"][1] == 0).all() and (got["scaled"][0][1] == 0).all() and (got["scaled"][1][1] == 0).all()
    y = O.as64(got["y"])
    assert np.isnan(y[3]).all() and np.isnan(y[2, 5])               # as the formula has it: inf * 0, nan
    v, _ = O.decode(got["scaled"], 400)
    assert np.isnan(v[3]).all() and np.isnan(v[2, 5])


def test_gradient_against_differences_of_the_kernel():
    x, r, gain, gy, gh = make(8, 600, torch.float32, 12)
    got = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True)
    back = api.tac_residual_norm_backward(got["h"], gain, got["rstd"], gy, gh)
    g = torch.Generator(device=DEV).manual_seed(13)
    dx, dg = torch.randn(8, 600, generator=g, device=DEV), torch.randn(600, generator=g, device=DEV)

    def loss(t):
        o = api.tac_residual_norm(x + t * dx, r, gain + t * dg, eps=EPS)
        return float((o["y"].double() * gy.double()).sum() + (o["h"].double() * gh.double()).sum())
    eps = 2.0 ** -7
    want = float((back["grad_x"].double() * dx.double()).sum() + (back["grad_gain"].double() * dg.double()).sum())
    # float32 values: each of the 9600 terms of the loss is off by at most about 2^-22 of its size (random signs: a hundred times that
    # at most), and the third derivative's share is eps^2 = 6e-5 of the terms' size; both are under 1 of the sum of sizes times 1e-4
    size = float((back["grad_x"].double() * dx.double()).abs().sum())
    assert abs((loss(eps) - loss(-eps)) / (2 * eps) - want) < 1e-3 * size


def test_on_another_stream_and_in_a_graph():
    x, r, gain, gy, gh = make(200, 1000, torch.bfloat16, 14)
    want = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True, want_scaled=True)
    want_back = api.tac_residual_norm_backward(want["h"], gain, want["rstd"], gy, gh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True, want_scaled=True, stream=side.cuda_stream)
    back = api.tac_residual_norm_backward(got["h"], gain, got["rstd"], gy, gh, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got["y"], want["y"]) and torch.equal(back["grad_x"], want_back["grad_x"])
    assert torch.equal(back["grad_gain"], want_back["grad_gain"])

    def both():
        o = api.tac_residual_norm(x, r, gain, eps=EPS, want_rstd=True, want_scaled=True)
        return o, api.tac_residual_norm_backward(o["h"], gain, o["rstd"], gy, gh)
    for o, b in O.captured(both):
        assert torch.equal(o["y"], want["y"]) and torch.equal(o["scaled"][0], want["scaled"][0])
        assert torch.equal(b["grad_x"], want_back["grad_x"]) and torch.equal(b["grad_gain"], want_back["grad_gain"])
        o["y"].zero_()
        b["grad_gain"].fill_(float("nan"))


def test_offsets_beyond_32_bits():
    rows, cols = 600_000, 4096                                   # 4.9 GB of bfloat16 each way
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    x.normal_()
    y = torch.empty_like(x)
    api.tac_residual_norm(x, None, None, eps=EPS, y=y)
    for at in (0, rows // 2, rows - 3):
        check_forward(x[at:at + 3], None, None, dict(h=None, y=y[at:at + 3], rstd=None, scaled=None))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 100, 400, 1001, 1300, 2049, 9000])
def test_pad_codes_are_zero_beside_infinities_and_nan(cols, dtype):
    x, _, gain, _, _ = make(5, cols, dtype, 15, residual=False)
    x[1, cols // 2], x[2, cols - 1], x[3, :] = float("nan"), float("inf"), -float("inf")
    scaled = api.tac_residual_norm(x, None, gain, eps=EPS, want_scaled=True)["scaled"]
    assert np.isnan(O.decode(scaled, cols)[0][[1, 3]]).all() and O.pads_are_zero(scaled, cols)
