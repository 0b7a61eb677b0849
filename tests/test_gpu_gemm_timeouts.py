"""hpsgd_gemm_fp8 in the checked build when its waits run out: what is reported, and that nothing is written or added."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests.test_gpu_gemm import BF, F32, Operand, check, product
from tests.test_gpu_ops_checked import checked_library  # noqa: F401

pytestmark = pytest.mark.gpu

# whole tiles; two, four and eight joined parts; pairs of SMs; parts that go through memory
FORMS = [(300, 600, 512), (1000, 1000, 2049), (100, 1100, 5000), (1, 256, 4096), (1300, 2100, 1700), (1, 100, 40000)]


@pytest.mark.parametrize("M,N,K", FORMS)
@pytest.mark.parametrize("out,accumulate", [(F32, False), (F32, True), (BF, False)])
def test_nothing_is_written(checked_library, M, N, K, out, accumulate):  # noqa: F811
    a, b = Operand(M, K, 1), Operand(N, K, 2)
    d = torch.randn(M, N, device="cuda").to(out)
    before = d.clone()
    hp.hpsgd_ops_debug_stall(1)
    with pytest.raises(hp.HpsgdError) as err:
        product(M, N, K, a, b, d, accumulate=accumulate)
    assert err.value.code == hp.HPSGD_E_TIMEOUT
    assert torch.equal(d, before)
    hp.hpsgd_ops_debug_stall(0)
    product(M, N, K, a, b, d, accumulate=accumulate)
    check(d, a, b, K, before if accumulate else None)


@pytest.mark.parametrize("M,N,K", [(1000, 1000, 2049), (100, 1100, 5000), (1, 256, 4096), (33, 200, 33000), (1, 100, 40000)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_one_missing_part_leaves_the_tile(checked_library, M, N, K, accumulate):  # noqa: F811
    """Only the blocks of odd numbers give up: every tile has parts of both kinds, and none of it may be written."""
    a, b = Operand(M, K, 1), Operand(N, K, 2)
    d = torch.randn(M, N, device="cuda")
    before = d.clone()
    hp.hpsgd_ops_debug_stall(2)
    with pytest.raises(hp.HpsgdError) as err:
        product(M, N, K, a, b, d, accumulate=accumulate)
    assert err.value.code == hp.HPSGD_E_TIMEOUT
    assert torch.equal(d, before)
    hp.hpsgd_ops_debug_stall(0)
    product(M, N, K, a, b, d, accumulate=accumulate)
    check(d, a, b, K, before if accumulate else None)


def test_whole_tiles_of_other_blocks_are_written(checked_library):  # noqa: F811
    """One tile a block: those of even numbers are complete, those of odd numbers untouched."""
    M, N, K = 16, 512, 256
    a, b = Operand(M, K, 1), Operand(N, K, 2)
    d = torch.full((M, N), 7.0, device="cuda")
    hp.hpsgd_ops_debug_stall(2)
    with pytest.raises(hp.HpsgdError) as err:
        product(M, N, K, a, b, d)
    assert err.value.code == hp.HPSGD_E_TIMEOUT
    hp.hpsgd_ops_debug_stall(0)
    want = torch.full((M, N), 7.0, device="cuda")
    whole = torch.empty(M, N, device="cuda")
    product(M, N, K, a, b, whole)
    for tile in (0, 2):
        want[:, tile * 128: tile * 128 + 128] = whole[:, tile * 128: tile * 128 + 128]
    assert torch.equal(d, want)
    with pytest.raises(hp.HpsgdError):
        hp.hpsgd_ops_debug_stall(3)
