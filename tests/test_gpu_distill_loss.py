"""hpsgd_distill_loss / _backward against the loss in binary64."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import loss_ref as ref

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
KIND = {F32: hp.HPSGD_F32, BF: hp.HPSGD_BF16}
HALF = {F32: 2.0 ** -24, BF: 2.0 ** -8}            # half a step, relative to the value
MARK = 77.0


class Case:
    def __init__(self, rows, vocab, k, T=1.0, wl=0.6, wt=0.4, dtype=F32, teacher_dtype=F32, labels=True, pad=0, shift=0, seed=0, spread=3.0):
        self.rows, self.vocab, self.k, self.T, self.wl, self.wt, self.dtype, self.ld = rows, vocab, k, T, wl, wt, dtype, vocab + pad
        g = torch.Generator().manual_seed(seed)

        def matrix(x):
            flat = torch.full((shift + rows * self.ld + 16,), MARK, dtype=dtype, device="cuda")
            view = flat[shift: shift + rows * self.ld].view(rows, self.ld)[:, :vocab]
            view.copy_(x.to(dtype))
            return view

        self.z = matrix(torch.randn(rows, vocab, generator=g) * spread + torch.randn(rows, 1, generator=g) * 5.0)
        self.dz = matrix(torch.full((rows, vocab), MARK))
        self.labels = torch.randint(0, vocab, (rows,), generator=g).cuda() if labels else None
        self.index = torch.stack([torch.randperm(vocab, generator=g)[:k] if k <= vocab else torch.randint(0, vocab, (k,), generator=g) for _ in range(rows)]).int().cuda() if k else None
        self.teacher = (torch.randn(rows, k, generator=g) * 2.0 + 3.0).to(teacher_dtype).cuda() if k else None
        self.dloss = (torch.rand(rows, generator=g) + 0.1).cuda()
        self.loss, self.lse = torch.full((rows + 1,), MARK, device="cuda"), torch.full((rows + 1, 2), MARK, device="cuda")

    def args(self, **change):
        kw = dict(logits=self.z, labels=self.labels, teacher_index=self.index, teacher_logits=self.teacher, temperature=self.T, label_weight=self.wl,
                  teacher_weight=self.wt, loss=self.loss, lse=self.lse, dlogits=self.dz, dloss=self.dloss, grad_scale=0.5, ldlogits=self.ld, lddlogits=self.ld)
        return hp.make_distill_loss(self.rows, self.vocab, self.k, KIND[self.dtype], **{**kw, **change})

    def check_gradient(self, dz, later):
        d = lambda x: x.double().cpu().numpy()  # noqa: E731
        z, dz, up = d(self.z), d(dz), d(self.dloss) * 0.5
        index = self.index.cpu().numpy() if self.k else np.zeros((self.rows, 0), int)
        teacher = d(self.teacher) if self.k else np.zeros((self.rows, 0))
        lse = d(self.lse)
        for r in range(self.rows):
            label = int(self.labels[r]) if self.labels is not None and self.wl > 0 else -1
            given = (lse[r, 0], lse[r, 1]) if later else None
            loss, one, two, grad, loss_err, lse_err, err = ref.row(z[r], label, index[r] if self.wt > 0 else [], teacher[r] if self.wt > 0 else [], self.T, self.wl, self.wt, given)
            if not later:
                assert abs(float(self.loss[r]) - loss) <= loss_err + 2.0 ** -23 * abs(loss) or float(self.loss[r]) == loss, (r, float(self.loss[r]), loss, loss_err)
                assert abs(lse[r, 0] - one) <= lse_err[0] and abs(lse[r, 1] - two) <= lse_err[1], (r, lse[r], one, two)
            want, e = grad * up[r], err * abs(up[r])
            off = np.abs(dz[r] - want) - e - HALF[self.dtype] * (np.abs(want) + e) - 2.0 ** -126
            assert (off <= 0).all(), (r, off.max(), np.argwhere(off > 0)[:5], later)

    def check(self):
        hp.hpsgd_distill_loss(self.args())
        torch.cuda.synchronize()
        assert float(self.loss[-1]) == MARK and bool((self.lse[-1] == MARK).all())
        self.check_gradient(self.dz, False)
        fused, loss, lse = self.dz.clone(), self.loss.clone(), self.lse.clone()
        self.dz.fill_(MARK)
        hp.hpsgd_distill_loss_backward(self.args(loss=None))
        torch.cuda.synchronize()
        self.check_gradient(self.dz, True)
        hp.hpsgd_distill_loss(self.args(dlogits=None, dloss=None))              # the loss alone
        assert torch.equal(self.loss, loss) and torch.equal(self.lse, lse)
        hp.hpsgd_distill_loss(self.args(loss=None, lse=None))                   # the gradient without them: there may be one temperature less
        torch.cuda.synchronize()
        self.check_gradient(self.dz, False)
        if self.ld > self.vocab:
            assert float((self.dz.as_strided((self.rows, self.ld - self.vocab), (self.ld, 1), self.dz.storage_offset() + self.vocab).float() - MARK).abs().max()) == 0.0
        assert float((self.dz._base[-16:].float() - MARK).abs().max()) == 0.0
        return fused


SHAPES = [(1, 1, 1), (3, 2, 0), (5, 7, 3), (4, 512, 8), (3, 1024, 130), (3, 1025, 5), (2, 4099, 64), (2, 8192, 17), (3, 8200, 4), (2, 16385, 33), (2, 30000, 64),
          (1, 65537, 9), (2, 131072, 32), (1, 131080, 3), (1, 262149, 5)]


@pytest.mark.parametrize("rows,vocab,k", SHAPES)
@pytest.mark.parametrize("dtype,T", [(F32, 1.0), (BF, 2.0), (F32, 0.7), (BF, 1.0)], ids=str)
def test_sizes(rows, vocab, k, dtype, T):
    Case(rows, vocab, k, T, dtype=dtype, teacher_dtype=BF if vocab % 2 else F32, seed=vocab + k).check()


@pytest.mark.parametrize("labels,wl,wt,k", [(True, 1.0, 0.0, 0), (True, 1.0, 0.0, 9), (False, 1.0, 1.0, 9), (True, 0.0, 1.0, 9), (False, 0.0, 1.0, 1024)])
@pytest.mark.parametrize("T", [1.0, 3.0])
def test_one_term_alone(labels, wl, wt, k, T):
    Case(3, 5000, k, T, wl, wt, labels=labels, dtype=BF, seed=k).check()
    Case(2, 20001, k, T, wl, wt, labels=labels, seed=k).check()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (0, 1), (3, 2), (0, 8)])
def test_strides_and_alignment(dtype, pad, shift):
    Case(4, 1000, 6, 2.0, dtype=dtype, pad=pad, shift=shift, seed=pad).check()
    Case(3, 20003, 6, 2.0, dtype=dtype, pad=pad, shift=shift, seed=pad).check()


@pytest.mark.parametrize("vocab", [600, 33000])
def test_entries_that_are_not_there_and_entries_twice(vocab):
    c = Case(8, vocab, 12, 2.0, seed=1)
    c.labels[1] = c.labels[3] = -100
    c.labels[7] = -(1 << 40)
    c.index[2, 4:] = -1
    c.index[3] = -1                                    # neither label nor teacher
    c.index[4] = c.labels[4].int()                     # all the same, and the label
    c.index[5, ::2] = c.index[5, 1]
    c.teacher[6] = float("-inf")                       # no teacher either
    c.teacher[7, 3:] = float("-inf")
    c.index[0, 0], c.index[0, 1], c.labels[0] = 0, vocab - 1, vocab - 1
    c.check()
    assert float(c.loss[3]) == 0.0 and float(c.dz[3].abs().max()) == 0.0
    c.z[3] = float("nan")
    hp.hpsgd_distill_loss(c.args())
    assert float(c.loss[3]) == 0.0 and float(c.dz[3].abs().max()) == 0.0


@pytest.mark.parametrize("vocab", [600, 33000])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_words_that_are_masked(vocab, T):
    c = Case(5, vocab, 10, T, seed=2)
    c.z[0, 5:] = float("-inf")
    c.z[0, 5:12] = 1.0
    c.index[0] = torch.arange(10)
    c.labels[0] = 11
    c.z[1] = torch.finfo(F32).min                      # masked by the lowest value, but for three
    c.z[1, 7:10] = torch.tensor([3.0, 1.0, 2.0])
    c.index[1] = -1
    c.index[1, :3] = torch.tensor([7, 8, 9])
    c.labels[1] = 8
    c.z[2] = 1e4 * c.z[2]                               # far apart
    c.z[3] = 0.0
    c.check()
    # a label or a teacher's entry on a masked word: an infinite loss, a finite gradient
    c.z[0, :] = float("-inf")
    c.z[0, :20] = torch.arange(20.0)
    c.labels[0], c.labels[4] = 30, -1
    c.z[4, 3] = float("-inf")
    c.index[4, 2] = 3
    hp.hpsgd_distill_loss(c.args())
    torch.cuda.synchronize()
    assert float(c.loss[0]) == float("inf") and float(c.loss[4]) == float("inf")
    assert bool(torch.isfinite(c.dz[0]).all()) and bool(torch.isfinite(c.dz[4]).all()) and float(c.dz[0, 31]) == 0.0


@pytest.mark.parametrize("vocab", [600, 33000])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_rows_that_are_wrong_are_nan_and_the_others_are_not(vocab, T):
    c = Case(9, vocab, 6, T, seed=3)
    c.labels[0] = vocab
    c.labels[1] = 1 << 40
    c.index[2, 3] = vocab
    c.index[3, 0] = 0x7FFFFFFF
    c.z[4, 17] = float("nan")
    c.z[5, 18] = float("inf")
    for later in (False, True):
        if later:
            c.dz.fill_(0.0)
            hp.hpsgd_distill_loss(Case.args(c, dlogits=None))
            c.lse[:4] = 1.0                             # (the sums of the first four were NaN)
            hp.hpsgd_distill_loss_backward(c.args())
        else:
            hp.hpsgd_distill_loss(c.args())
            assert bool(torch.isnan(c.loss[:6]).all()) and bool(torch.isfinite(c.loss[6:9]).all())
        torch.cuda.synchronize()
        assert bool(torch.isnan(c.dz[:6]).all()) and bool(torch.isfinite(c.dz[6:]).all())
    c.dloss[:6] = 0.0                                   # rows that count for nothing
    hp.hpsgd_distill_loss(c.args())
    assert float(c.dz[:6].abs().max()) == 0.0 and float(c.dz[6:].abs().max()) > 0.0


@pytest.mark.parametrize("vocab,dtype", [(700, F32), (20003, BF), (300001, BF), (9000, F32)])
def test_in_place_the_same_bits_and_from_a_graph(vocab, dtype):
    c = Case(3, vocab, 20, 2.0, dtype=dtype, seed=4)
    hp.hpsgd_distill_loss(c.args())
    first, loss = c.dz.clone(), c.loss.clone()
    keep = c.z.clone()
    hp.hpsgd_distill_loss(c.args(dlogits=c.z))
    assert torch.equal(c.z, first) and torch.equal(c.loss, loss)
    c.z.copy_(keep)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hp.hpsgd_distill_loss(c.args())
        hp.hpsgd_distill_loss_backward(c.args(dlogits=c.dz))
    c.z.copy_(keep.flip(0))
    for name in ("labels", "index", "teacher", "dloss"):
        getattr(c, name).copy_(getattr(c, name).flip(0).clone())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.loss[:3], loss[:3].flip(0))
    c.check_gradient(c.dz, True)


def test_many_rows_and_offsets_beyond_2_to_the_31():
    rows, vocab = 72_000, 32_000
    z = torch.zeros(rows, vocab, dtype=BF, device="cuda")
    labels = torch.randint(0, vocab, (rows,), device="cuda")
    loss = torch.empty(rows, device="cuda")
    hp.hpsgd_distill_loss(hp.make_distill_loss(rows, vocab, 0, hp.HPSGD_BF16, z, labels=labels, loss=loss, dlogits=z))
    torch.cuda.synchronize()
    # uniform: log(32000) = 10.3735; its bound as in the reference
    assert float((loss - float(np.log(32000.0))).abs().max()) < 1e-5
    p = torch.tensor(1.0 / vocab).to(BF)
    at = torch.arange(rows, device="cuda")
    assert bool((z[at, labels] == torch.tensor(1.0 / vocab - 1.0).to(BF).cuda()).all())
    z[at, labels] = p.cuda()
    assert bool((z[-3:] == p.cuda()).all()) and bool((z[rows // 2] == p.cuda()).all())
