"""hpsgd_gated_ffn_forward in the checked build: the same results, and when its waits run out, what is reported, and that nothing is written."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests.test_gpu_gated_ffn import Forward, inputs
from tests.test_gpu_ops_checked import checked_library  # noqa: F401

pytestmark = pytest.mark.gpu

# whole tiles, one and several a block, on each width; two, four and eight joined parts
FORMS = [(16, 512, 256), (60, 300, 500), (300, 600, 512), (3000, 2000, 300), (100, 5000, 2000), (1, 2000, 1100), (5, 40, 16384)]


@pytest.mark.parametrize("M,N,K", FORMS)
@pytest.mark.parametrize("stall", [1, 2])
def test_nothing_is_written(checked_library, M, N, K, stall):  # noqa: F811
    """Stall 2: blocks of odd numbers alone give up; a tile in parts then has parts of both kinds."""
    c = Forward(M, N, K, "silu", *inputs(M, N, K, 1))
    before = [x.clone() for x in (c.z, c.gu, c.z8.q, c.z8.s)]
    hp.hpsgd_ops_debug_stall(stall)
    with pytest.raises(hp.HpsgdError) as err:
        c.run()
    assert err.value.code == hp.HPSGD_E_TIMEOUT and "hpsgd_gated_ffn_forward" in str(err.value)
    hp.hpsgd_ops_debug_stall(0)
    if stall == 1 or (M, N, K) in FORMS[-3:]:
        assert all(torch.equal(x, y) for x, y in zip(before, (c.z, c.gu, c.z8.q, c.z8.s)))
    c.run()
    c.check()
