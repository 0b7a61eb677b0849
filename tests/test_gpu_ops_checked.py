"""The operators in the checked build: the product's bounded waits run out when they are made to, and everything carries on."""
import time

import pytest
import torch

import paper_2009_02701_b200 as hp
from paper_2009_02701_b200 import build
from tests.test_gpu_gemm import Operand, check, product

pytestmark = pytest.mark.gpu


@pytest.fixture
def checked_library():
    hp.hpsgd_destroy()
    hp.use_library(build.build(debug=True))
    try:
        yield
    finally:
        hp.hpsgd_ops_debug_stall(0)
        hp.use_library(None)


@pytest.mark.parametrize("M,N,K", [(1, 256, 512), (300, 600, 512), (1, 256, 4096), (1300, 2100, 1700)], ids=["two blocks", "blocks", "joined blocks", "pairs"])
def test_waits_that_run_out(checked_library, M, N, K):
    a, b = Operand(M, K, 1), Operand(N, K, 2)
    d = torch.zeros(M, N, device="cuda")
    product(M, N, K, a, b, d)
    check(d, a, b, K)
    hp.hpsgd_ops_debug_stall(1)
    start = time.monotonic()
    with pytest.raises(hp.HpsgdError) as err:
        product(M, N, K, a, b, d)
    assert err.value.code == hp.HPSGD_E_TIMEOUT and time.monotonic() - start < 20.0
    hp.hpsgd_ops_debug_stall(0)
    for _ in range(3):                      # reported once; the device and the tensor memory are as before
        d.zero_()
        product(M, N, K, a, b, d)
        check(d, a, b, K)
