"""hpsgd_gemm_fp8 at the lower end of binary32: subnormal results, and subnormal values in what is added to."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests.test_gpu_gemm import F32, Operand, product

pytestmark = pytest.mark.gpu

# whole tiles, joined parts, pairs of SMs, parts that go through memory
FORMS = [(3, 200, 256), (100, 300, 4096), (1300, 2100, 1700), (3, 100, 40000)]


def ones(rows, cols, byte_a):
    """A matrix of ones in the block format times 2^(byte - 127)."""
    x = Operand(rows, cols, 1, spread=0)
    x.q[:, :cols] = 0x38
    x.s[:] = byte_a
    return x


@pytest.mark.parametrize("M,N,K", FORMS)
def test_nothing_added_changes_nothing(M, N, K):
    """D += 0 for D of every size, subnormal values among them."""
    a, b = Operand(M, K, 3), Operand(N, K, 4)
    a.q[:, :K] = 0
    g = torch.Generator(device="cuda").manual_seed(1)
    bits = torch.randint(0, 0x7F800000, (M, N), generator=g, device="cuda", dtype=torch.int32)
    bits[:, ::3] &= 0x7FFFFF                     # subnormal
    d = bits.view(F32).clone()
    d[::2] *= -1.0
    before = d.clone()
    product(M, N, K, a, b, d, accumulate=True)
    assert torch.equal(d.view(torch.int32), before.view(torch.int32))


@pytest.mark.parametrize("M,N,K", FORMS)
def test_sums_of_normal_numbers_that_are_subnormal(M, N, K):
    """K ones times 2^-125 / 2^ceil(log2 K): exact sums between 2^-126 and 2^-125, of which D takes away all but a few units of 2^-149."""
    up = (K - 1).bit_length()
    a, b = ones(M, K, 127 - 61 - up), ones(N, K, 127 - 64)
    want = K * 2.0 ** (-125 - up)                # every partial sum is exact: K < 2^24
    d = torch.empty(M, N, device="cuda")
    product(M, N, K, a, b, d)
    assert bool((d.double() == want).all())
    left = torch.arange(N, device="cuda", dtype=torch.float64).remainder(9.0) * 2.0 ** -149
    d = (-want + left).to(F32).expand(M, N).contiguous()
    assert torch.equal(d[0].double(), -want + left)      # binary32 holds it: the sum's last unit is 2^-149
    product(M, N, K, a, b, d, accumulate=True)
    assert torch.equal(d.double(), left.expand(M, N))


@pytest.mark.parametrize("M,N,K", FORMS)
def test_subnormal_products(M, N, K):
    """K ones times 2^-145: sums that are subnormal as long as K is below 2^19."""
    a, b = ones(M, K, 127 - 75), ones(N, K, 127 - 70)
    want = K * 2.0 ** -145
    d = torch.empty(M, N, device="cuda")
    product(M, N, K, a, b, d)
    assert bool((d.double() == want).all())
    d.fill_(2.0 ** -140)
    product(M, N, K, a, b, d, accumulate=True)
    assert bool((d.double() == want + 2.0 ** -140).all())
