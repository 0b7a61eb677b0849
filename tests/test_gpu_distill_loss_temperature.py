"""hpsgd_distill_loss / _backward at temperatures far above and below 1, where the two softmaxes have little in common."""
import pytest
import torch

from tests import test_gpu_distill_loss as ordinary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [100.0, 130.0, 200.0, 1e3, 1e6, 0.05, 1e-3])
@pytest.mark.parametrize("vocab,dtype", [(600, ordinary.F32), (9000, ordinary.BF), (33000, ordinary.F32)], ids=str)
def test_a_largest_logit_that_comes_late(vocab, dtype, T):
    """A step of the softened softmax's exponent is T log 2 logits wide; the other's has to move on its own."""
    c = ordinary.Case(4, vocab, 7, T, dtype=dtype, seed=vocab)
    for r in range(3):
        c.z[r] = torch.linspace(-5.0, 10.0, vocab, device="cuda").flip(0) if r else 10.0
        c.z[r, vocab - 40 * (r + 1)] = 130.0
    c.check()
