"""hpsgd_ops_check where waits ran out in more than one operator and on more than one stream: all of it is reported, and once."""
import gc
import time

import pytest
import torch

import paper_2009_02701_b200 as hp
from tests.test_gpu_gated_ffn import Forward, inputs
from tests.test_gpu_gemm import Operand
from tests.test_gpu_ops_checked import checked_library  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def nothing_left():
    """A caught time-out holds its frames, and they the operands: both are let go here, not whenever the collector comes by, so that they do not cut up the device
    memory that later tests get."""
    yield
    gc.collect()


class Product:
    def __init__(self, M, N, K):
        self.a, self.b, self.d = Operand(M, K, 1), Operand(N, K, 2), torch.zeros(M, N, device="cuda")
        self.workspace = torch.zeros(16 + hp.hpsgd_gemm_fp8_bytes(M, N, K), dtype=torch.uint8, device="cuda")
        self.args = hp.make_gemm_fp8(M, N, K, self.a.q, self.a.s, self.b.q, self.b.s, self.d, hp.HPSGD_F32, workspace=self.workspace)


def test_both_operators_are_named(checked_library):  # noqa: F811
    p, layer = Product(300, 600, 512), Forward(60, 300, 500, "silu", *inputs(60, 300, 500, 1))
    call = layer.args()
    torch.cuda.synchronize()
    hp.hpsgd_ops_debug_stall(1)
    hp.hpsgd_gemm_fp8(p.args)
    hp.hpsgd_gated_ffn_forward(call)
    with pytest.raises(hp.HpsgdError) as err:
        hp.hpsgd_ops_check()
    hp.hpsgd_ops_debug_stall(0)
    assert err.value.code == hp.HPSGD_E_TIMEOUT
    assert "hpsgd_gemm_fp8" in str(err.value) and "hpsgd_gated_ffn_forward" in str(err.value)
    hp.hpsgd_ops_check()


@pytest.mark.parametrize("first", ["product", "layer"])
def test_a_report_takes_in_the_other_streams(checked_library, first):  # noqa: F811
    """One stream's call has given up when it is asked after; the other's is still waiting, and gives up during the report."""
    p, layer = Product(300, 600, 512), Forward(60, 300, 500, "silu", *inputs(60, 300, 500, 1))
    call = layer.args()
    one, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    hp.hpsgd_ops_debug_stall(1)
    run = [lambda s: hp.hpsgd_gemm_fp8(p.args, s), lambda s: hp.hpsgd_gated_ffn_forward(call, s)]
    run[first == "layer"](one)
    time.sleep(1.0)
    run[first != "layer"](other)
    with pytest.raises(hp.HpsgdError) as err:
        hp.hpsgd_ops_check(one)
    hp.hpsgd_ops_debug_stall(0)
    assert err.value.code == hp.HPSGD_E_TIMEOUT
    assert "hpsgd_gemm_fp8" in str(err.value) and "hpsgd_gated_ffn_forward" in str(err.value)
    hp.hpsgd_ops_check(other)
