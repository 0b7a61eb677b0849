"""Refusals of the gated feed-forward layer: error codes before any GPU work, so all of it runs without a device."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp

A = 1 << 20            # an address that is aligned for everything; nothing is ever read from it


def refused(code, call, *args, **kw):
    with pytest.raises(hp.HpsgdError) as err:
        call(*args, **kw)
    assert err.value.code == code, str(err.value)


def forward(M=5, N=100, K=200, act=0, **kw):
    return hp.make_gated_ffn_forward(M, N, K, act, **{**dict(x=A, x_scale=A, w=A, w_scale=A, z8=A, z_scale=A, z=A, gu=A), **kw})


def backward(M=5, N=100, act=0, **kw):
    return hp.make_gated_ffn_backward(M, N, act, **{**dict(gu=A, dz=A, dz_dtype=0, dq=A, dq_scale=A, dqt=A, dqt_scale=A, dgu=2 * A), **kw})


@pytest.mark.parametrize("change", [dict(M=-1), dict(N=-1), dict(K=-1), dict(K=0), dict(act=2), dict(act=-1), dict(z_dtype=2), dict(x=None), dict(w=None), dict(x_scale=None),
                                    dict(w_scale=None), dict(z8=None), dict(z_scale=None), dict(z8=None, z_scale=None, z=None), dict(x=A + 8), dict(w=A + 8), dict(z8=A + 8),
                                    dict(x_scale=A + 2), dict(w_scale=A + 2), dict(z_scale=A + 2), dict(z=A + 1), dict(z=A + 2, z_dtype=0), dict(gu=A + 1), dict(ldx=200),
                                    dict(ldx=192), dict(ldw=192), dict(ldsx=4), dict(ldsw=199), dict(ldz8=96), dict(ldz8=120), dict(ldsz=4), dict(ldz=99), dict(ldgu=199)], ids=str)
def test_forward_refuses(change):
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_gated_ffn_forward(forward(**change)))


@pytest.mark.parametrize("change", [dict(M=-1), dict(N=-1), dict(act=2), dict(dz_dtype=2), dict(gu=None), dict(dz=None), dict(dq=None), dict(dq_scale=None), dict(dqt=None),
                                    dict(dqt_scale=None), dict(dq=None, dq_scale=None, dqt=None, dqt_scale=None, dgu=None), dict(gu=A + 1), dict(dz=A + 2), dict(dgu=A + 1),
                                    dict(dz=A + 1, dz_dtype=1), dict(dq=A + 8), dict(dqt=A + 8), dict(dq_scale=A + 2), dict(dqt_scale=A + 2), dict(ldgu=199), dict(lddz=99),
                                    dict(lddgu=199), dict(lddq=192), dict(lddqt=8), dict(ldsdq=4), dict(ldsdqt=199), dict(dgu=A)], ids=str)
def test_backward_refuses(change):
    refused(hp.HPSGD_E_BADARG, lambda: hp.hpsgd_gated_ffn_backward(backward(**change)))


def test_sizes():
    for change in (dict(M=1 << 31), dict(N=1 << 30), dict(K=1 << 31)):
        refused(hp.HPSGD_E_UNSUPPORTED, lambda: hp.hpsgd_gated_ffn_forward(forward(**change)))
    for change in (dict(M=1 << 31), dict(N=1 << 30)):
        refused(hp.HPSGD_E_UNSUPPORTED, lambda: hp.hpsgd_gated_ffn_backward(backward(**change)))
    for change in (dict(M=0), dict(N=0)):
        assert hp.hpsgd_gated_ffn_forward(forward(**change)) == 0 and hp.hpsgd_gated_ffn_backward(backward(**change)) == 0
    with pytest.raises(TypeError):
        forward(ldu=4)


def test_arguments_take_no_host_memory():
    for make, names in ((forward, "x x_scale w w_scale z8 z_scale z gu"), (backward, "gu dz dq dq_scale dqt dqt_scale dgu")):
        make()
        for name in names.split():
            for host in (torch.zeros(1 << 12), np.zeros(1 << 12, np.float32)):
                refused(hp.HPSGD_E_BADARG, make, **{name: host})


@pytest.mark.gpu
def test_arguments_are_checked_tensors():
    z = lambda *s, dtype=torch.uint8: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    BF, F32 = torch.bfloat16, torch.float32
    good = dict(x=z(5, 208), x_scale=z(1, 5, 4), w=z(200, 208), w_scale=z(1, 200, 4), z8=z(5, 112), z_scale=z(1, 5, 4), z=z(5, 100, dtype=BF), gu=z(5, 200, dtype=BF))
    forward(**{**good, "z_dtype": 1})
    for name, bad in (("x", z(5, 208, dtype=F32)), ("x", z(4, 208)), ("x_scale", z(1, 4, 4)), ("w", z(199, 208)), ("w_scale", z(1, 199, 4)), ("z8", z(5, 96)), ("z_scale", z(1, 4, 4)),
                      ("z", z(5, 100, dtype=F32)), ("z", z(4, 100, dtype=BF)), ("gu", z(5, 100, dtype=BF)), ("gu", z(5, 200, dtype=torch.float16))):
        refused(hp.HPSGD_E_BADARG, forward, **{**good, "z_dtype": 1, name: bad})
    good = dict(gu=z(5, 200, dtype=BF), dz=z(5, 100, dtype=F32), dq=z(5, 208), dq_scale=z(1, 5, 4), dqt=z(200, 16), dqt_scale=z(1, 200, 4), dgu=z(5, 200, dtype=BF))
    backward(**good)
    for name, bad in (("gu", z(5, 200, dtype=F32)), ("dz", z(5, 100, dtype=BF)), ("dq", z(5, 192)), ("dq_scale", z(1, 4, 4)), ("dqt", z(199, 16)), ("dqt_scale", z(1, 199, 4)), ("dgu", z(5, 199, dtype=BF))):
        refused(hp.HPSGD_E_BADARG, backward, **{**good, name: bad})
