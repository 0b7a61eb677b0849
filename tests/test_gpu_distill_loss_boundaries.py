"""Logits and their gradient on different boundaries: groups of eight that lie alike in neither are put together from aligned pieces."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import test_gpu_distill_loss as ordinary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [ordinary.F32, ordinary.BF])
@pytest.mark.parametrize("vocab,T", [(5, 1.0), (1000, 2.0), (9001, 1.5), (20004, 1.0), (131075, 3.0)])
@pytest.mark.parametrize("of_z,of_dz,pad", [(0, 1, 0), (3, 0, 5), (2, 6, 1), (0, 0, 4)])
def test_they_may_differ(dtype, vocab, T, of_z, of_dz, pad):
    """of_z, of_dz: elements behind a wide boundary; pad: elements between the gradient's rows."""
    c, rows = ordinary.Case(3, vocab, min(vocab, 6), T, dtype=dtype, shift=of_z, seed=vocab + of_z), 3
    flat = torch.full((of_dz + rows * (vocab + pad) + 16,), ordinary.MARK, dtype=dtype, device="cuda")
    dz = flat[of_dz: of_dz + rows * (vocab + pad)].view(rows, vocab + pad)
    for later in (False, True):
        flat.fill_(ordinary.MARK)
        (hp.hpsgd_distill_loss_backward if later else hp.hpsgd_distill_loss)(c.args(dlogits=dz[:, :vocab], lddlogits=vocab + pad))
        torch.cuda.synchronize()
        c.check_gradient(dz[:, :vocab], later)
        around = torch.cat([flat[:of_dz], dz[:, vocab:].reshape(-1), flat[-16:]])
        assert bool((around == ordinary.MARK).all())
