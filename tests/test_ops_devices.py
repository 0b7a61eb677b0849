"""Argument blocks whose tensors are on another device than the current one, or on several: refused before a kernel could read them from there.  (Needs
no device: the tensors say where they are, and nothing of them is read.)"""
import pytest
import torch

import paper_2009_02701_b200 as hp
from paper_2009_02701_b200 import binding, ops


class Elsewhere:
    """A matrix of floats as the binding sees it."""
    is_cuda = True

    def __init__(self, device, rows, cols, dtype=torch.float32):
        self.device, self.like = device, torch.empty(rows, cols, dtype=dtype, device="meta")
        self.shape, self.dtype = self.like.shape, dtype

    def __getattr__(self, name):
        return getattr(self.like, name)

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 1 << 20


class Library:
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        return lambda *args: self.called.append(name) or 0


def scan(first, others):
    m = lambda d: Elsewhere(d, 12, 16)  # noqa: E731
    return hp.make_gated_scan_forward(12, 16, 3, hp.HPSGD_F32, m(first), m(others), m(others))


def loss(first, others):
    return hp.make_distill_loss(4, 32, 0, hp.HPSGD_F32, Elsewhere(first, 4, 32), dlogits=Elsewhere(others, 4, 32))


@pytest.mark.parametrize("make,call", [(scan, hp.hpsgd_gated_scan_forward), (loss, hp.hpsgd_distill_loss), (loss, hp.hpsgd_distill_loss_backward)])
def test_tensors_elsewhere(monkeypatch, make, call):
    library, there, here = Library(), make(1, 1), make(0, 0)
    with pytest.raises(hp.HpsgdError) as err:
        make(1, 0)
    assert err.value.code == hp.HPSGD_E_BADARG and "device" in str(err.value)
    monkeypatch.setattr(binding, "_lib", library)
    monkeypatch.setattr(ops, "_current_device", lambda: 0)
    for stream in (None, 0, 12345):
        with pytest.raises(hp.HpsgdError) as err:
            call(there, stream)
        assert err.value.code == hp.HPSGD_E_BADARG and "device 1" in str(err.value)
    assert not library.called
    call(here, 0)
    assert len(library.called) == 1
