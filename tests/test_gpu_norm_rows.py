"""The norm with more rows than blocks are resident: the forward pass's forms for many rows, the backward pass's loop over rows."""
import pytest
import torch

from tests.test_gpu_norm import BF, F32, test_backward as backward, test_forward as forward

pytestmark = pytest.mark.gpu

# 1184 rows and more take two groups a thread (up to 4096 columns): 64, 128 and 256 threads a row, each at both ends of its widths, with widths
# that leave the second group partly or wholly empty, on and off the wide boundary
MANY = [(1184, 513), (1185, 520), (1185, 1023), (1184, 1024), (1200, 1032), (1185, 2007), (1184, 2048), (1190, 2056), (1184, 4090), (1185, 4096), (1184, 300),
        (1190, 8185), (1184, 8200)]


@pytest.mark.parametrize("rows,cols", MANY)
@pytest.mark.parametrize("dtype,wdtype", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("residual", [True, False])
def test_forward_of_many_rows(rows, cols, dtype, wdtype, residual):
    forward(rows, cols, dtype, wdtype, residual)


# Every width of a row's threads, and rows enough for a second, a third and an uneven last turn of the grid
TURNS = [(9500, 100), (4800, 300), (1300, 1000), (2400, 1024), (1300, 2008), (1185, 2007), (700, 4096), (1000, 4090), (330, 8200), (330, 8185), (310, 16384),
         (450, 6001), (593, 2048)]


@pytest.mark.parametrize("rows,cols", TURNS)
@pytest.mark.parametrize("dtype,wdtype", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("residual", [True, False])
def test_backward_over_several_turns(rows, cols, dtype, wdtype, residual):
    backward(rows, cols, dtype, wdtype, residual)
