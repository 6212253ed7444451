"""8-bit matrices: bit for bit against the definition."""
import numpy as np
import pytest
import torch

import head_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]
SHAPES = [(1, 1), (1, 128), (128, 1), (3, 130), (127, 129), (128, 128), (200, 513), (300, 640), (65, 1100), (520, 257)]


def make(rows, cols, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    v = torch.randn(rows, cols, generator=g, device=DEV) * torch.exp(3 * torch.randn(rows, 1, generator=g, device=DEV))
    return (v * torch.exp(torch.randn(cols, generator=g, device=DEV))).to(dtype)


def check(matrix, want, e_want, cols):
    v, e = O.decode(matrix, cols)
    assert np.array_equal(e, e_want)
    assert np.array_equal(v, want, equal_nan=True)
    assert O.pads_are_zero(matrix, cols)


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rows_and_columns(rows, cols, dtype, tiles):
    x = make(rows, cols, dtype, 200 + rows)
    got = api.tac_quantize(x, tiles=tiles, rows=True, columns=True)
    x64 = O.as64(x)
    check(got["rows"], *O.quantized(x64, tiles), cols)
    check(got["columns"], *O.quantized(np.ascontiguousarray(x64.T), tiles), rows)
    for only in (dict(rows=True, columns=False), dict(rows=False, columns=True)):
        one = api.tac_quantize(x, tiles=tiles, **only)
        for k in ("rows", "columns"):
            if only[k]:
                assert torch.equal(one[k][0], got[k][0]) and torch.equal(one[k][1], got[k][1])
            else:
                assert one[k] is None
    if tiles:                                                    # a matrix in tiles and its transpose are the same numbers
        assert np.array_equal(O.decode(got["rows"], cols)[0], O.decode(got["columns"], rows)[0].T)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_an_8bit_matrix_laid_out_again(rows, cols):
    kept = api.tac_quantize(make(rows, cols, torch.float32, 300 + cols))["rows"]
    values, e = O.decode(kept, cols)
    got = api.tac_quantize(kept, cols=cols, rows=True, columns=True)
    check(got["rows"], *O.quantized(values), cols)
    check(got["columns"], *O.quantized(np.ascontiguousarray(values.T)), rows)
    assert np.array_equal(O.decode(got["rows"], cols)[0], values)           # along the rows nothing changes


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_back_to_floats_is_exact(rows, cols, dtype):
    kept = api.tac_quantize(make(rows, cols, torch.float32, 400 + cols))["rows"]
    values, _ = O.decode(kept, cols)
    assert np.array_equal(O.as64(api.tac_dequantize(kept, cols, dtype=dtype)), values)
    wide = torch.full((rows, cols + 3), float("nan"), dtype=dtype, device=DEV)
    api.tac_dequantize(kept, cols, out=wide[:, :cols])
    assert np.array_equal(O.as64(wide[:, :cols]), values) and torch.isnan(wide[:, cols:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("move", ["strided", "shifted"])
def test_strides_and_addresses(dtype, move):
    x = make(140, 264, dtype, 5)
    want = api.tac_quantize(x, columns=True)
    got = api.tac_quantize(O.strided(x, 3) if move == "strided" else O.shifted(x), columns=True)
    for k in ("rows", "columns"):
        assert torch.equal(got[k][0], want[k][0]) and torch.equal(got[k][1], want[k][1])


@pytest.mark.parametrize("dtype", TYPES)
def test_borders_zeros_infinities_nan_and_the_smallest(dtype):
    x = torch.zeros(12, 200, dtype=dtype, device=DEV)
    x[1, 3] = 448.0
    x[2, 3] = 450.0                                              # just beyond the largest code: the next scale
    x[3, 3] = -448.0 * 2.0 ** 40
    x[4, 7], x[4, 8], x[4, 9] = float("inf"), 3.0, -float("inf")
    x[5, 130], x[5, 131] = float("nan"), 1e-3
    x[6, :] = 2.0 ** -130                                        # below the smallest scale's subnormals in part
    x[7, 0], x[7, 1] = 3.0e38, 1.0
    x[8, :] = float("nan")
    x[9, :] = torch.arange(200, device=DEV) * 2.0 ** -126
    x[10, 0], x[10, 1] = 1.0, 2.0 ** -12                         # ties in the subnormals
    x[11, ::2] = -0.0
    x64 = O.as64(x)
    got = api.tac_quantize(x, columns=True)
    check(got["rows"], *O.quantized(x64), 200)
    check(got["columns"], *O.quantized(np.ascontiguousarray(x64.T)), 12)


def test_every_bfloat16_number():
    bits = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16)
    x = bits.view(torch.bfloat16).reshape(512, 128)
    got = api.tac_quantize(x, columns=True)
    x64 = O.as64(x)
    check(got["rows"], *O.quantized(x64), 128)
    check(got["columns"], *O.quantized(np.ascontiguousarray(x64.T)), 512)


def test_on_another_stream_and_in_a_graph():
    x = make(300, 700, torch.bfloat16, 6)
    want = api.tac_quantize(x, columns=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = api.tac_quantize(x, columns=True, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got["columns"][0], want["columns"][0])
    for g in O.captured(lambda: api.tac_quantize(x, columns=True)):
        for k in ("rows", "columns"):
            assert torch.equal(g[k][0], want[k][0]) and torch.equal(g[k][1], want[k][1])
        g["rows"][0].zero_()
        g["columns"][0].zero_()


def test_offsets_beyond_32_bits():
    rows, cols = 1_100_000, 4096                                  # 4.5 GB of codes
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    x.normal_()
    got = api.tac_quantize(x, columns=True)
    for at in (0, rows - 130):
        check((got["rows"][0][at:at + 130], got["rows"][1][at:at + 130]), *O.quantized(O.as64(x[at:at + 130])), cols)
    for c in (0, cols - 2):                                       # the last block of the transposed rows, from a multiple of 128 on
        r0 = rows // 128 * 128
        want, e = O.quantized(np.ascontiguousarray(O.as64(x[r0:, c:c + 2]).T))
        codes, scales = got["columns"][0][c:c + 2, r0:], got["columns"][1][c:c + 2, r0 // 128:]
        check((codes.contiguous(), scales.contiguous()), want, e, rows - r0)
    back = api.tac_dequantize(got["rows"], cols, dtype=torch.bfloat16)
    assert np.array_equal(O.as64(back[rows - 2:]), O.decode((got["rows"][0][rows - 2:], got["rows"][1][rows - 2:]), cols)[0])


def test_more_tiles_than_512_threads_each_fit_a_launch():
    square = 1 << 15
    x = torch.empty((1, square * square + 200), dtype=torch.bfloat16, device=DEV)        # 2^23 + 2 tiles of one row
    x.normal_()
    codes, scales = api.tac_quantize(x)["rows"]
    want = api.tac_quantize(x[:, :square * square].view(square, square))["rows"]
    assert torch.equal(codes[:, :square * square].view(square, square), want[0])
    assert torch.equal(scales[:, :square * square // 128].view(square, -1), want[1])
    check((codes[:, square * square:].contiguous(), scales[:, square * square // 128:].contiguous()), *O.quantized(O.as64(x[:, square * square:])), 200)
