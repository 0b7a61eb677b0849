"""Refusals of the loss: error codes before any GPU work, so all of it runs without a device."""
import math

import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp

A = 1 << 20            # an address that is aligned for everything; nothing is ever read from it


def refused(code, call, *args, **kw):
    with pytest.raises(hp.HpsgdError) as err:
        call(*args, **kw)
    assert err.value.code == code, str(err.value)


def make(rows=5, vocab=100, k=3, dtype=0, **kw):
    return hp.make_distill_loss(rows, vocab, k, dtype, **{**dict(logits=A, labels=A, teacher_index=A, teacher_logits=A, loss=A, lse=A, dlogits=2 * A, dloss=A,
                                                                 teacher_weight=1.0), **kw})


@pytest.mark.parametrize("change", [dict(rows=-1), dict(vocab=-1), dict(k=-1), dict(dtype=2), dict(teacher_dtype=7), dict(temperature=0.0), dict(temperature=-1.0),
                                    dict(temperature=math.nan), dict(temperature=math.inf), dict(temperature=1e-30), dict(temperature=1e30), dict(label_weight=-1.0),
                                    dict(label_weight=math.inf), dict(teacher_weight=math.nan), dict(teacher_weight=-0.5), dict(teacher_weight=1e38, temperature=10.0),
                                    dict(grad_scale=math.inf), dict(grad_scale=math.nan), dict(logits=None), dict(teacher_index=None), dict(teacher_logits=None),
                                    dict(logits=A + 2), dict(labels=A + 4), dict(teacher_index=A + 2), dict(teacher_logits=A + 2), dict(loss=A + 1), dict(lse=A + 2),
                                    dict(dlogits=A + 2), dict(dloss=A + 3), dict(ldlogits=99), dict(lddlogits=99), dict(ldteacher=2), dict(ldlogits=-100),
                                    dict(dlogits=A, ldlogits=104), dict(logits=A + 1, dtype=1), dict(teacher_logits=A + 1, teacher_dtype=1)], ids=str)
def test_both_refuse(change):
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_distill_loss(make(**change)))
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_distill_loss_backward(make(**change)))


def test_outputs_and_sizes():
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_distill_loss(make(loss=None, lse=None, dlogits=None)))
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_distill_loss_backward(make(dlogits=None)))
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_distill_loss_backward(make(lse=None)))
    for call in (hp.hpsgd_distill_loss, hp.hpsgd_distill_loss_backward):
        for change in (dict(k=1025), dict(vocab=1 << 31), dict(rows=1 << 30)):
            refused(hp.HPSGD_E_UNSUPPORTED, lambda: call(make(**change)))
        for change in (dict(rows=1 << 31), dict(rows=1 << 62), dict(rows=(1 << 62) + 5), dict(rows=(1 << 63) - 1, vocab=1)):
            refused(hp.HPSGD_E_UNSUPPORTED, lambda: call(make(**change)))
        for change in (dict(rows=0), dict(vocab=0)):
            assert call(make(**change)) == 0
    with pytest.raises(TypeError):
        make(ldlabels=4)


def test_arguments_take_no_host_memory():
    make()
    for name in "logits labels teacher_index teacher_logits loss lse dlogits dloss".split():
        for host in (torch.zeros(1 << 12), np.zeros(1 << 12, np.float32)):
            refused(hp.HPSGD_E_BADARG, make, **{name: host})


@pytest.mark.gpu
def test_arguments_are_checked_tensors():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    good = dict(logits=z(5, 100), labels=z(5, dtype=torch.int64), teacher_index=z(5, 3, dtype=torch.int32), teacher_logits=z(5, 3), loss=z(5), lse=z(5, 2), dlogits=z(5, 100), dloss=z(5))
    make(**good)
    make(**{**good, "teacher_logits": z(5, 3, dtype=torch.bfloat16)})          # its type is the tensor's
    for name, bad in (("logits", z(5, 100, dtype=torch.bfloat16)), ("logits", z(4, 100)), ("logits", z(5, 200)[:, ::2]), ("labels", z(5, dtype=torch.int32)), ("labels", z(4, dtype=torch.int64)),
                      ("teacher_index", z(5, 3, dtype=torch.int64)), ("teacher_index", z(4, 3, dtype=torch.int32)), ("teacher_logits", z(5, 3, dtype=torch.float16)),
                      ("teacher_logits", z(14)), ("loss", z(4)), ("lse", z(9)), ("dlogits", z(5, 100, dtype=torch.float64)), ("dloss", z(5, 2)[:, 0])):
        refused(hp.HPSGD_E_BADARG, make, **{**good, name: bad})
