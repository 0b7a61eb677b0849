"""The widest rows that the gated recurrence takes: a block's columns behind the last are counted in 32 bits too."""
import pytest

import paper_2009_02701_b200 as hp
from tests.test_gated_scan_host import backward, forward, refused

WIDEST = (1 << 31) - 1 - 512


@pytest.mark.parametrize("cols", [WIDEST + 1, (1 << 31) - 300, (1 << 31) - 65])
def test_rows_that_are_too_wide(cols):
    refused(hp.HPSGD_E_UNSUPPORTED, lambda: hp.hpsgd_gated_scan_forward(forward(cols=cols)))
    refused(hp.HPSGD_E_UNSUPPORTED, lambda: hp.hpsgd_gated_scan_forward(forward(cols=cols, rows=3)))
    refused(hp.HPSGD_E_UNSUPPORTED, lambda: hp.hpsgd_gated_scan_backward(backward(cols=cols)))
    assert hp.hpsgd_gated_scan_saved_bytes(8, cols) == 0 and hp.hpsgd_gated_scan_saved_bytes(8, WIDEST) == (WIDEST + 3) // 4 * 16
