"""Refusals of the gated recurrence: error codes before any GPU work, so all of it runs without a device."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp

A = 1 << 20            # an address that is aligned for everything; nothing is ever read from it


def refused(code, call, *args, **kw):
    with pytest.raises(hp.HpsgdError) as err:
        call(*args, **kw)
    assert err.value.code == code, str(err.value)


def forward(rows=12, cols=10, sequences=3, dtype=0, **kw):
    return hp.make_gated_scan_forward(rows, cols, sequences, dtype, **{**dict(f=A, v=A, o=A, y=A, h0=A, h_last=A, saved=A), **kw})


def backward(rows=12, cols=10, sequences=3, dtype=0, **kw):
    return hp.make_gated_scan_backward(rows, cols, sequences, dtype, **{**dict(f=A, v=A, o=A, do=A, saved=A, dy=A, df=A, dv=A, h0=A, dh0=A, dh_last=A), **kw})


@pytest.mark.parametrize("change", [dict(rows=-3), dict(cols=-1), dict(sequences=-1), dict(dtype=2), dict(dtype=-1), dict(rows=13), dict(f=None), dict(v=None),
                                    dict(y=None), dict(offsets=A + 4), dict(f=A + 2), dict(v=A + 1), dict(o=A + 2), dict(y=A + 2), dict(saved=A + 8), dict(h0=A + 2),
                                    dict(h_last=A + 2), dict(ldf=9), dict(ldv=9), dict(ldo=9), dict(ldy=9), dict(ldh0=9), dict(ldlast=9), dict(ldf=-10),
                                    dict(ldh0=11), dict(f=A + 1, dtype=1)], ids=str)
def test_forward_refuses(change):
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_gated_scan_forward(forward(**change)))


@pytest.mark.parametrize("change", [dict(rows=-3), dict(cols=-1), dict(sequences=-1), dict(dtype=2), dict(rows=13), dict(f=None), dict(v=None), dict(saved=None),
                                    dict(dy=None), dict(df=None), dict(dv=None), dict(do=None), dict(o=None), dict(offsets=A + 4), dict(f=A + 2), dict(v=A + 2),
                                    dict(o=A + 2), dict(dy=A + 2), dict(df=A + 2), dict(dv=A + 2), dict(do=A + 2), dict(saved=A + 8), dict(h0=A + 2),
                                    dict(dh0=A + 2), dict(dh_last=A + 2), dict(ldf=9), dict(ldv=9), dict(ldo=9), dict(lddy=9), dict(lddf=9), dict(lddv=9),
                                    dict(lddo=9), dict(ldh0=9), dict(lddh0=9), dict(lddlast=9)], ids=str)
def test_backward_refuses(change):
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_gated_scan_backward(backward(**change)))


def test_sizes():
    for make, call in ((forward, hp.hpsgd_gated_scan_forward), (backward, hp.hpsgd_gated_scan_backward)):
        for change in (dict(rows=1 << 31, sequences=1), dict(cols=1 << 31), dict(sequences=1 << 31, offsets=A)):
            refused(hp.HPSGD_E_UNSUPPORTED, lambda: call(make(**change)))
        for change in (dict(cols=0), dict(sequences=0)):          # nothing to do
            assert call(make(**change)) == 0
    assert hp.hpsgd_gated_scan_forward(forward(rows=0, h_last=None)) == 0 and hp.hpsgd_gated_scan_backward(backward(rows=0, dh0=None)) == 0
    assert hp.hpsgd_gated_scan_saved_bytes(0, 5) == hp.hpsgd_gated_scan_saved_bytes(5, 0) == hp.hpsgd_gated_scan_saved_bytes(-1, 5) == 0
    assert hp.hpsgd_gated_scan_saved_bytes(1, 5) == 32 and hp.hpsgd_gated_scan_saved_bytes(17, 5) == 96
    with pytest.raises(TypeError):
        forward(ldsaved=4)


def test_arguments_take_no_host_memory():
    for make, names in ((forward, "f v o y offsets h0 h_last saved"), (backward, "f v o do saved dy df dv h0 dh0 dh_last offsets")):
        make()
        for name in names.split():
            for host in (torch.zeros(1 << 12), np.zeros(1 << 12, np.float32)):
                refused(hp.HPSGD_E_BADARG, make, **{name: host})


@pytest.mark.gpu
def test_arguments_are_checked_tensors():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    good = dict(f=z(12, 10), v=z(12, 10), o=z(12, 10), y=z(12, 10), h0=z(3, 10), h_last=z(3, 10), saved=z(24), offsets=z(4, dtype=torch.int64))
    forward(**good)
    for name, bad in (("f", z(12, 10, dtype=torch.bfloat16)), ("v", z(11, 10)), ("o", z(12, 20)[:, ::2]), ("y", z(10, 12).t()), ("h0", z(2, 10)), ("h_last", z(3, 10, dtype=torch.float16)),
                      ("saved", z(23)), ("offsets", z(4, dtype=torch.int32)), ("offsets", z(3, dtype=torch.int64))):
        refused(hp.HPSGD_E_BADARG, forward, **{**good, name: bad})
    good = dict(f=z(12, 10), v=z(12, 10), o=z(12, 10), do=z(12, 10), saved=z(24), dy=z(12, 10), df=z(12, 10), dv=z(12, 10), h0=z(3, 10), dh0=z(3, 10), dh_last=z(3, 10))
    backward(**good)
    for name, bad in (("do", z(11, 10)), ("dy", z(12, 10, dtype=torch.bfloat16)), ("df", z(119)), ("dv", z(12, 11)[:, :10]), ("dh0", z(29)), ("dh_last", z(2, 10)), ("saved", z(23))):
        refused(hp.HPSGD_E_BADARG, backward, **{**good, name: bad})
