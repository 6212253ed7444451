"""Products of 8-bit matrices on every tile of the kernel: in one round of workgroups, in several, in parts of the columns."""
import pytest
import torch

from paper_2603_13810_amd import api
from test_gpu_product import check, matrix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# bfloat16 results, tile, M, N, K, parts, more than one round (asserted on the CPU by test_product_plan.py)
CASES = [(0, 0, 5518, 2181, 266, 1, False), (0, 0, 6313, 3998, 279, 1, True), (0, 0, 6154, 669, 10240, 3, False),
         (0, 2, 3075, 1295, 266, 1, False), (0, 2, 4083, 2324, 262, 1, True), (0, 2, 283, 6555, 9471, 3, False),
         (0, 3, 6314, 455, 269, 1, False), (0, 3, 1411, 5377, 266, 1, True), (0, 3, 2753, 1, 3994, 16, False),
         (0, 7, 45, 42, 279, 1, False), (0, 7, 658, 5634, 263, 1, True), (0, 7, 1, 1, 1677, 6, False),
         (1, 0, 2200, 3771, 263, 1, False), (1, 0, 4368, 6012, 262, 1, True), (1, 0, 6541, 589, 8728, 3, False),
         (1, 1, 4995, 594, 391, 1, False), (1, 1, 65, 2724, 10014, 8, False),
         (1, 2, 1584, 2599, 267, 1, False), (1, 2, 6703, 2463, 283, 1, True), (1, 2, 5520, 140, 9678, 4, False),
         (1, 4, 6608, 263, 279, 1, False), (1, 4, 4611, 1674, 289, 1, True),
         (1, 5, 132, 5636, 281, 1, False), (1, 5, 1, 647, 10751, 32, False),
         (1, 6, 73, 4411, 263, 1, False), (1, 6, 1, 323, 6067, 24, False),
         (1, 8, 46, 41, 262, 1, False), (1, 8, 33, 8170, 513, 1, False), (1, 8, 40, 700, 5000, 8, False)]


def values(m, cols):
    """The float64 values of an 8-bit matrix, bit by bit, on the GPU."""
    codes, scales = m[0].to(torch.int32), m[1]
    x, f = (codes >> 3) & 15, (codes & 7).double()
    v = torch.where(x == 0, f * 2.0 ** -9, (8 + f) * torch.exp2(x.double() - 10)) * torch.where(codes >= 128, -1.0, 1.0)
    return (v * torch.exp2(scales.double() - 127).repeat_interleave(128, 1)[:, :v.shape[1]])[:, :cols]


@pytest.mark.parametrize("bf16,t,M,N,K,parts,rounds", CASES)
def test_tile(bf16, t, M, N, K, parts, rounds):
    a, b = matrix(M, K, 31), matrix(N, K, 32)
    bias = torch.randn(N, device=DEV)
    dtype = torch.bfloat16 if bf16 else torch.float32
    a64, b64 = values(a, K), values(b, K)
    y, size = a64 @ b64.t() + bias.double(), a64.abs() @ b64.abs().t() + bias.double().abs()
    got = api.tac_scaled_product(*a, *b, K, bias=bias, dtype=dtype)
    check(got, y, size, K)
    for _ in range(3):                       # workgroups go on from item to item: nothing of one may reach the next
        assert torch.equal(got, api.tac_scaled_product(*a, *b, K, bias=bias, dtype=dtype))
    odd = torch.full((M, N + 3), float("nan"), dtype=dtype, device=DEV)
    api.tac_scaled_product(*a, *b, K, bias=bias, out=odd[:, 1:N + 1])      # rows that start anywhere
    assert torch.equal(odd[:, 1:N + 1], got) and bool(torch.isnan(odd[:, [0, N + 1, N + 2]]).all())
    plain = api.tac_scaled_product(*a, *b, K, dtype=dtype)
    check(plain, y - bias.double(), size, K)
