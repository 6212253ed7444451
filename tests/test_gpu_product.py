"""Products of 8-bit matrices against 64 bits."""
import numpy as np
import pytest
import torch

import head_util as O
from paper_2603_13810_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]


def matrix(rows, cols, seed, tiles=False, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    v = torch.randn(rows, cols, generator=g, device=DEV) * torch.exp(spread * torch.randn(rows, 1, generator=g, device=DEV))
    v *= torch.exp(spread * torch.randn(cols, generator=g, device=DEV))
    return api.tac_quantize(v, tiles=tiles)["rows"]


def exact(a, b, K, bias=None):
    """The product and the sum of its terms' magnitudes, 64 bits (on the GPU, from values decoded on the CPU for small sizes)."""
    a64, b64 = (torch.from_numpy(O.decode(m, K)[0]).to(DEV) for m in (a, b))
    y, size = a64 @ b64.t(), a64.abs() @ b64.t().abs()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, size


def check(got, y, size, K):
    # codes multiply exactly; sums of K terms in float32, at worst one rounding (here: truncation, 2^-23) a term, of at most the
    # sum of magnitudes; then the rounding of the output.  bfloat16 output: the 8-bit instruction adds eight products at a time and drops
    # what is below 2^-13 of the largest of them (seen by giving it 2^16 and one smaller term), which is in `size` too
    tol = O.HALF[got.dtype] * y.abs() + (K + 20) * 2 * O.U * size
    if got.dtype == torch.bfloat16:
        tol = tol + 7 * 2.0 ** -13 * size
    assert bool(((got.double() - y).abs() <= tol * (1 + 1e-6)).all()), float(((got.double() - y).abs() / (tol + 1e-300)).max())


SHAPES = [(1, 1, 1), (1, 16, 128), (3, 5, 100), (16, 16, 129), (17, 33, 512), (20, 48, 640), (31, 100, 1000), (64, 64, 256), (65, 127, 385),
          (128, 128, 128), (130, 260, 700), (256, 256, 1024), (257, 300, 513), (500, 129, 2049), (1000, 520, 384), (12, 700, 9000), (700, 12, 9000),
          (40, 40, 33000), (300, 4100, 256), (2048, 2048, 300)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_against_64_bits(M, N, K, dtype):
    a, b = matrix(M, K, 1), matrix(N, K, 2)
    bias = torch.randn(N, device=DEV) if (M + N) % 2 else None
    got = api.tac_scaled_product(*a, *b, K, bias=bias, dtype=dtype)
    y, size = exact(a, b, K, bias)
    check(got, y, size, K)
    assert torch.equal(got, api.tac_scaled_product(*a, *b, K, bias=bias, dtype=dtype))        # no order of arrival
    wide = torch.full((M, N + 5), float("nan"), dtype=dtype, device=DEV)
    api.tac_scaled_product(*a, *b, K, bias=bias, out=wide[:, :N])
    assert torch.equal(wide[:, :N], got) and bool(torch.isnan(wide[:, N:]).all())


@pytest.mark.parametrize("M,N,K", [(5, 40, 700), (300, 260, 700), (600, 700, 1400)])
def test_every_place_has_its_own_value(M, N, K):
    # one term per place, a different power of two or small whole number for each row, column and block: any row, column, block
    # or byte that is taken for another shows up exactly
    a, b = torch.zeros(M, K, device=DEV), torch.zeros(N, K, device=DEV)
    rows, cols = torch.arange(M, device=DEV), torch.arange(N, device=DEV)
    for k in range(0, K, 37):
        a[rows, (k + rows) % K] = (1 + rows % 7) * 2.0 ** ((k // 128 + rows) % 7 - 3)
        b[cols, (k + 3 * cols) % K] = (1 + cols % 15) * 2.0 ** ((k // 128 + 2 * cols) % 7 - 3)
    qa, qb = api.tac_quantize(a)["rows"], api.tac_quantize(b)["rows"]
    y, size = exact(qa, qb, K)
    got = api.tac_scaled_product(*qa, *qb, K, dtype=torch.float32)
    # terms are multiples of 2^-6, and their magnitudes add up to less than 2^18: every partial sum is a float32 number
    assert float(size.max()) < 2.0 ** 18 and torch.equal(got.double(), y)


@pytest.mark.parametrize("M", [1, 17, 300])
def test_nan_stays_in_its_row_and_column(M):
    N, K = 150, 600
    a, b = torch.randn(M, K, device=DEV), torch.randn(N, K, device=DEV)
    a[M - 1, 500], b[7, 3] = float("nan"), float("inf")
    qa, qb = api.tac_quantize(a)["rows"], api.tac_quantize(b)["rows"]
    got = torch.isnan(api.tac_scaled_product(*qa, *qb, K, dtype=torch.float32))
    want = torch.zeros_like(got)
    want[M - 1], want[:, 7] = True, True
    assert torch.equal(got, want)


def test_smallest_and_largest_scales():
    K = 256
    a, b = torch.randn(40, K, device=DEV) * 2.0 ** 100, torch.randn(50, K, device=DEV) * 2.0 ** -100
    qa, qb = api.tac_quantize(a)["rows"], api.tac_quantize(b)["rows"]
    y, size = exact(qa, qb, K)
    check(api.tac_scaled_product(*qa, *qb, K, dtype=torch.float32), y, size, K)


@pytest.mark.parametrize("rows,cols,n", [(70, 300, 200), (520, 384, 640), (900, 129, 257)])
def test_the_three_products_of_a_dense_layer(rows, cols, n):
    g = torch.Generator(device=DEV).manual_seed(4)
    x, w, gy = (torch.randn(*s, generator=g, device=DEV) for s in ((rows, cols), (n, cols), (rows, n)))
    qx, qw, qg = api.tac_quantize(x)["rows"], api.tac_quantize(w, tiles=True, columns=True), api.tac_quantize(gy, columns=True)
    x64, w64, g64 = (torch.from_numpy(O.decode(m, c)[0]).to(DEV) for m, c in ((qx, cols), (qw["rows"], cols), (qg["rows"], n)))
    f32 = torch.float32
    check(api.tac_scaled_product(*qx, *qw["rows"], cols, dtype=f32), x64 @ w64.t(), x64.abs() @ w64.abs().t(), cols)
    # the transposed weights hold the same values as the weights
    check(api.tac_scaled_product(*qg["rows"], *qw["columns"], n, dtype=f32), g64 @ w64, g64.abs() @ w64.abs(), n)
    kept = api.tac_quantize(qx, cols=cols, rows=False, columns=True)["columns"]
    gt, xt = (torch.from_numpy(O.decode(m, rows)[0]).to(DEV) for m in (qg["columns"], kept))
    check(api.tac_scaled_product(*qg["columns"], *kept, rows, dtype=f32), gt @ xt.t(), gt.abs() @ xt.abs().t(), rows)


@pytest.mark.parametrize("M,N,K", [(9, 300, 2000), (300, 200, 700), (64, 64, 20000)])
def test_on_another_stream_and_in_a_graph(M, N, K):
    a, b = matrix(M, K, 5), matrix(N, K, 6)
    want = api.tac_scaled_product(*a, *b, K)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = api.tac_scaled_product(*a, *b, K, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want)
    for g in O.captured(lambda: api.tac_scaled_product(*a, *b, K)):
        assert torch.equal(g, want)
        g.zero_()


@pytest.mark.parametrize("M", [7, 300])
def test_offsets_beyond_32_bits(M):
    N, K = 150_000, 32768                                          # 4.9 GB of codes
    codes = torch.randint(0, 120, (N, K), dtype=torch.uint8, device=DEV)
    scales = torch.randint(110, 130, (N, 4 * (-(-K // 512))), dtype=torch.uint8, device=DEV)
    a = matrix(M, K, 7)
    got = api.tac_scaled_product(*a, codes, scales, K, dtype=torch.float32)
    for at in (0, N - 70):
        y, size = exact(a, (codes[at:at + 70], scales[at:at + 70]), K)
        check(got[:, at:at + 70], y, size, K)


def test_output_beyond_32_bits():
    M, N, K = 70_000, 20_000, 128                                   # 5.6 GB of float32
    a, b = matrix(M, K, 8), matrix(N, K, 9)
    got = api.tac_scaled_product(*a, *b, K, dtype=torch.float32)
    y, size = exact((a[0][-50:], a[1][-50:]), b, K)
    check(got[-50:], y, size, K)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 40, 700), (5, 40, 700), (70, 260, 900), (300, 260, 700), (600, 700, 1400), (2200, 1500, 300)])
def test_one_product_per_place_is_exact(M, N, K, dtype):
    # every row of a has one value, so a place is one product of two numbers of four bits: exact in bfloat16 too, whichever instruction multiplies.
    # Values differ by row, column, block and byte
    a, rows, cols, k = torch.zeros(M, K, device=DEV), torch.arange(M, device=DEV), torch.arange(N, device=DEV), torch.arange(K, device=DEV)
    a[rows, 37 * rows % K] = (1 + rows % 15) * 2.0 ** (rows % 9 - 4)
    b = (1 + (cols[:, None] + 3 * k[None, :]) % 15) * 2.0 ** ((2 * cols[:, None] + k[None, :] // 128) % 11 - 5)
    qa, qb = api.tac_quantize(a)["rows"], api.tac_quantize(b)["rows"]
    want = a[rows, 37 * rows % K].double()[:, None] * b.double()[:, 37 * rows % K].t()
    assert torch.equal(api.tac_scaled_product(*qa, *qb, K, dtype=dtype).double(), want)


@pytest.mark.parametrize("M", [1, 20, 300])
@pytest.mark.parametrize("spread", [0.0, 1.0])
@pytest.mark.parametrize("N,K", [(2000, 512), (2000, 4096), (300, 20000)])
def test_digits_of_the_8bit_instruction(M, N, K, spread):
    # The bias takes the sum away again, so that the bfloat16 result is the sum's error (one row of a, M times).
    g = torch.Generator(device=DEV).manual_seed(41)
    scale = torch.exp(spread * torch.randn(2, K, generator=g, device=DEV))
    a, b = torch.randn(1, K, generator=g, device=DEV) * scale[0], torch.randn(N, K, generator=g, device=DEV) * scale[1]
    qa, qb = api.tac_quantize(a)["rows"], api.tac_quantize(b)["rows"]
    terms = torch.from_numpy(O.decode(qa, K)[0] * O.decode(qb, K)[0]).to(DEV)
    y = terms.sum(1)
    got = api.tac_scaled_product(*(t.expand(M, -1).contiguous() for t in qa), *qb, K, bias=-y.float())
    assert all(torch.equal(got[i], got[0]) for i in range(M))
    error = (got[0].double() - (y - y.float().double())) / (1 + O.HALF[torch.bfloat16])
    # eight neighbours lose less than 2^-13 of the largest each; signs are mixed, so errors up to q of either sign add up to at most
    # sqrt(8 / 3) q per eight in the root mean square, over all eights
    q = 2.0 ** -13 * torch.nn.functional.pad(terms, (0, -K % 8)).abs().view(N, -1, 8).amax(2)
    f32 = K * O.U * y.abs().max()                        # sums in float32 and the bias's rounding, far below
    assert bool((error.abs() <= 8 * q.sum(1) + f32).all())
    assert float(error.square().mean()) <= 8 / 3 * float(q.square().sum(1).mean()) + float(f32) ** 2
    # what tac.h states of a sum: a relative error of a few 1e-5 (and not float32's 6e-8 either, which this instruction does not have)
    assert float(error.square().mean().sqrt() / y.square().mean().sqrt()) < 1e-4


@pytest.mark.parametrize("dtype", TYPES)
def test_the_largest_numbers_are_2_to_the_128(dtype):
    # as tac.h has it: between the two last codes of the largest scale, 240 * 2^120 and 256 * 2^120, half way is 248 * 2^120 = 31/32 * 2^128
    low, high = 2.0 ** 128 * 30.75 / 32, torch.finfo(dtype).max
    a = torch.tensor([[high, 0.0], [low, 0.0], [-high, 1.0]], device=DEV, dtype=dtype)
    b = torch.tensor([[2.0 ** -100, 0.0], [0.0, 1.0]], device=DEV)
    qa, qb = api.tac_quantize(a)["rows"], api.tac_quantize(b)["rows"]
    assert O.decode(qa, 2)[0].tolist() == [[2.0 ** 128, 0.0], [240 * 2.0 ** 120, 0.0], [-2.0 ** 128, 0.0]]        # 1.0 is far below 2^120
    inf = float("inf")
    assert api.tac_dequantize(qa, 2, dtype=dtype).tolist() == [[inf, 0.0], [240 * 2.0 ** 120, 0.0], [-inf, 0.0]]
    assert api.tac_scaled_product(*qa, *qb, 2).tolist() == [[2.0 ** 28, 0.0], [240 * 2.0 ** 20, 0.0], [-2.0 ** 28, 0.0]]
    wide = api.tac_scaled_product(*qa, *qb, 2, dtype=torch.float32)
    assert wide[:, 0].tolist() == [inf, 240 * 2.0 ** 20, -inf] and wide[:, 1].isnan().tolist() == [True, False, True]
