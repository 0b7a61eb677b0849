"""Sequences without rows where blocks work in clusters: the half warps that pass their states on have different numbers of them."""
import pytest

from tests import test_gpu_gated_scan as ordinary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("empty", [1, 2, 5, 37, 300])
@pytest.mark.parametrize("cols", [64, 37])
@pytest.mark.parametrize("dtype,gate", [(ordinary.F32, False), (ordinary.BF, True)], ids=["f32", "bf16"])
def test_their_states_go_through(cols, dtype, gate, empty):
    for bounds in ([0] * (empty + 1) + [3000], [0, 2999] + [2999] * empty + [3000], [0] + [1500] * (empty + 1) + [3000] * 2):
        ordinary.Case(3000, cols, len(bounds) - 1, bounds=bounds, dtype=dtype, gate=gate, seed=empty).check()
