"""hpsgd_distill_loss / _backward where logits are masked by finite values, or so large that their exponents fill a binary32 number."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import loss_far_ref as ref
from tests import test_gpu_distill_loss as ordinary

pytestmark = pytest.mark.gpu

BF, F32, HALF = ordinary.BF, ordinary.F32, ordinary.HALF
LOWEST = {F32: float(torch.finfo(F32).min), BF: float(torch.finfo(BF).min)}
MASKS = [LOWEST[F32], LOWEST[BF], -1e30, -1e10, -4e6]


class Case(ordinary.Case):
    def check(self):
        """In one pass, later, and without a gradient."""
        hp.hpsgd_distill_loss(self.args())
        torch.cuda.synchronize()
        assert float(self.loss[-1]) == ordinary.MARK and bool((self.lse[-1] == ordinary.MARK).all())
        self.check_gradient(self.dz, False)
        loss, lse = self.loss.clone(), self.lse.clone()
        self.dz.fill_(ordinary.MARK)
        hp.hpsgd_distill_loss_backward(self.args(loss=None))
        torch.cuda.synchronize()
        self.check_gradient(self.dz, True)
        hp.hpsgd_distill_loss(self.args(dlogits=None, dloss=None))
        for x, y in ((self.loss, loss), (self.lse, lse)):
            torch.testing.assert_close(x, y, rtol=0.0, atol=0.0, equal_nan=True)
        hp.hpsgd_distill_loss(self.args(loss=None, lse=None))                   # there may be one temperature less
        torch.cuda.synchronize()
        self.check_gradient(self.dz, False)
        assert float((self.dz._base[-16:].float() - ordinary.MARK).abs().max()) == 0.0

    def check_gradient(self, dz, later):
        d = lambda x: x.double().cpu().numpy()  # noqa: E731
        z, dz, up, lse = d(self.z), d(dz), d(self.dloss) * 0.5, d(self.lse)
        index = self.index.cpu().numpy() if self.k else np.zeros((self.rows, 0), int)
        teacher = d(self.teacher) if self.k else np.zeros((self.rows, 0))
        for r in range(self.rows):
            if np.isposinf(z[r]).any():                # (a product that was too large for the stored type)
                assert np.isnan(dz[r]).all() and (later or np.isnan(float(self.loss[r])))
                continue
            label = int(self.labels[r]) if self.labels is not None and self.wl > 0 else -1
            loss, one, two, grad, loss_err, lse_err, err = ref.row(z[r], label, index[r] if self.wt > 0 else [], teacher[r] if self.wt > 0 else [], self.T, self.wl, self.wt,
                                                                   lse[r] if later else None)
            if not later:
                got = float(self.loss[r])
                assert abs(got - loss) <= loss_err + 2.0 ** -23 * abs(loss) or (got == float("inf") and loss > 2.0 ** 127), (r, got, loss, loss_err)
                for x, want, e in zip(lse[r], (one, two), lse_err):
                    with np.errstate(over="ignore"):
                        assert abs(x - want) <= e or x == float(np.float32(want)), (r, x, want, e)
            want, e = grad * up[r], err * abs(up[r])
            off = np.abs(dz[r] - want) - e - HALF[self.dtype] * (np.abs(want) + e) - 2.0 ** -126
            assert (off <= 0).all(), (r, off.max(), np.argwhere(off > 0)[:5], later)


def masked(vocab, mask, T, dtype, teacher_dtype=F32, seed=0):
    """Rows that are masked in different places."""
    mask, k = max(mask, LOWEST[dtype], LOWEST[teacher_dtype]), 6
    c = Case(12, vocab, k, T, dtype=dtype, teacher_dtype=teacher_dtype, seed=seed)
    z, index, teacher, labels = c.z, c.index, c.teacher, c.labels
    z[0, :300] = mask                                  # what some warps see first, or all that they see
    labels[0] = vocab - 1
    index[0] = torch.arange(k, device="cuda") + 400
    z[1, 3:] = mask
    z[2, :-3] = mask
    for r, first in ((1, 0), (2, vocab - 3)):          # the teacher's list is longer than what is allowed
        index[r] = torch.arange(k, device="cuda") + (first if r == 1 else vocab - 6)
        labels[r] = first + 1
        allowed = (index[r] >= first) & (index[r] < first + 3)
        teacher[r] = torch.where(allowed, teacher[r].float(), torch.tensor(mask, device="cuda")).to(teacher_dtype)
    z[3, 1::2] = mask
    index[3], labels[3] = torch.arange(k, device="cuda") * 2, 4
    teacher[4, 2] = mask
    teacher[5, 1:] = mask
    teacher[6] = mask                                  # all alike
    z[7] = mask                                        # nothing is left: all alike
    z[8], labels[8], index[8] = mask, -1, -1
    z[9] = mask
    teacher[9] = mask
    z[10, 17], labels[10] = mask, 17                   # a label that is masked: a large loss
    z[11, 18] = mask
    index[11] = torch.arange(k, device="cuda") + 14    # and a teacher's entry
    return c


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("T", [0.7, 1.0, 1.5, 2.0, 3.0, 4.0, 10.0])
@pytest.mark.parametrize("vocab,dtype", [(600, F32), (600, BF), (33000, F32), (33000, BF)], ids=str)
def test_words_that_are_masked_by_a_finite_value(vocab, dtype, T, mask):
    masked(vocab, mask, T, dtype, BF if vocab == 600 else F32, seed=vocab).check()


@pytest.mark.parametrize("mask", [LOWEST[BF], -1e10])
@pytest.mark.parametrize("T", [1.0, 2.0, 1.5])
def test_long_rows_and_rows_on_other_boundaries(mask, T):
    masked(131075, mask, T, BF, seed=1).check()
    c = masked(9001, mask, T, F32, seed=2)
    dz = torch.empty(12 * 9001 + 1, device="cuda")[1:].view(12, 9001)           # off the boundaries that the logits lie on
    hp.hpsgd_distill_loss(c.args(dlogits=dz))
    c.check_gradient(dz, False)
    dz.zero_()
    hp.hpsgd_distill_loss_backward(c.args(dlogits=dz))
    c.check_gradient(dz, True)


@pytest.mark.parametrize("labels,wl,wt", [(True, 1.0, 0.0), (False, 0.0, 1.0)])
@pytest.mark.parametrize("T", [1.0, 3.0, 1.5])
@pytest.mark.parametrize("mask", [LOWEST[F32], -1e10])
def test_one_term_alone(labels, wl, wt, T, mask):
    c = masked(2000, mask, T, F32, seed=4)
    c.wl, c.wt = wl, wt
    if not labels:
        c.labels = None
    c.check()


@pytest.mark.parametrize("scale", [1e6, 3e7, 1e12, 2e37])
@pytest.mark.parametrize("T", [1e-6, 0.5, 1.0, 2.0, 1.5])
def test_logits_that_are_large_all_over(scale, T):
    """Differences of a few units where the logits' own spacing allows them, and rows of both signs."""
    for vocab, dtype in ((700, F32), (20000, BF)):
        c = Case(6, vocab, 5, T, dtype=dtype, seed=6, spread=3.0)
        c.z[0] *= scale
        c.z[1] = c.z[1] * 0.5 + scale
        c.z[2] = c.z[2] * 0.5 - scale
        c.z[3] = scale
        c.z[3, 9] = -scale
        c.teacher[4] = c.teacher[4] * scale
        c.teacher[5] = c.teacher[5] - scale
        c.check()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_in_place_is_the_same_and_from_a_graph(dtype):
    for T, vocab in ((1.0, 40000), (2.5, 700), (2.0, 131075)):
        c = masked(vocab, LOWEST[BF], T, dtype, seed=8)
        hp.hpsgd_distill_loss(c.args())
        want, loss, z = c.dz.clone(), c.loss.clone(), c.z.clone()
        hp.hpsgd_distill_loss(c.args(dlogits=c.z))
        torch.cuda.synchronize()
        assert torch.equal(c.z, want) and torch.equal(c.loss, loss)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hp.hpsgd_distill_loss(c.args())
        c.z.copy_(z)
        c.dz.zero_()
        c.loss.fill_(ordinary.MARK)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.dz, want) and torch.equal(c.loss, loss)


def test_in_place_later_is_the_same():
    """The gradient alone, over the logits, where it starts from the logits and not from lse: several blocks would share such a row."""
    for T in (1.0, 2.5):
        c = masked(40000, LOWEST[F32], T, F32, seed=8)
        hp.hpsgd_distill_loss(c.args())
        hp.hpsgd_distill_loss_backward(c.args())
        want = c.dz.clone()
        hp.hpsgd_distill_loss_backward(c.args(dlogits=c.z))
        torch.cuda.synchronize()
        assert torch.equal(c.z, want) and bool(torch.isfinite(want).all())


def test_nan_and_infinity_stay_nan():
    for T in (1.0, 2.0, 1.5):
        c = Case(6, 5000, 4, T, seed=9)
        c.z[0] = float("nan")
        c.z[1] = LOWEST[F32]
        c.z[1, 77] = float("nan")
        c.z[2] = 1e30
        c.z[2, 4000] = float("inf")
        c.z[3] = -1e30
        c.labels[3] = 5000                             # outside the vocabulary
        c.z[4] = 1e30
        c.index[4, 1] = 5000
        hp.hpsgd_distill_loss(c.args())
        torch.cuda.synchronize()
        assert bool(torch.isnan(c.loss[:5]).all()) and bool(torch.isnan(c.dz[:5]).all()) and bool(torch.isfinite(c.loss[5:]).all()) and bool(torch.isfinite(c.dz[5]).all())
        c.dz.zero_()
        hp.hpsgd_distill_loss_backward(c.args())
        torch.cuda.synchronize()
        assert bool(torch.isnan(c.dz[:5]).all()) and bool(torch.isfinite(c.dz[5]).all())
        c.dloss[:5] = 0.0
        hp.hpsgd_distill_loss(c.args())
        assert float(c.dz[:5].abs().max()) == 0.0
