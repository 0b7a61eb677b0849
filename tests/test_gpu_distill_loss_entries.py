"""Teacher's entries that are not there: a logit of -infinity, or a negative index, whatever stands in the other place."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import test_gpu_distill_loss as ordinary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("index", [0, 1, 1 << 30, 0x7FFFFFFF], ids=["vocab", "vocab + 1", "2^30", "2^31 - 1"])
@pytest.mark.parametrize("vocab,dtype", [(600, ordinary.F32), (33000, ordinary.BF)], ids=str)
@pytest.mark.parametrize("T", [1.0, 2.0, 1.5])
def test_an_index_outside_the_vocabulary_with_no_logit(vocab, dtype, T, index):
    c = ordinary.Case(4, vocab, 9, T, dtype=dtype, seed=vocab)
    pad = index if index > 1 else vocab + index
    c.index[0, 5:], c.teacher[0, 5:] = pad, float("-inf")
    c.index[1], c.teacher[1] = pad, float("-inf")      # the label alone
    c.index[2], c.teacher[2], c.labels[2] = pad, float("-inf"), -1
    c.index[3, ::2], c.teacher[3, ::2] = -5, float("nan")
    c.check()
    assert float(c.loss[2]) == 0.0 and float(c.dz[2].abs().max()) == 0.0
    c.teacher[0, 7] = 1.0                              # there, and wrong
    hp.hpsgd_distill_loss(c.args())
    torch.cuda.synchronize()
    assert bool(torch.isnan(c.loss[0])) and bool(torch.isnan(c.dz[0]).all()) and bool(torch.isfinite(c.loss[1:4]).all())
