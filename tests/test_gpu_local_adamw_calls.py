"""hpsgd_local_step_adamw as a call of the library: its launches are profiled like every other step's, and a refusal enqueues nothing."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests.gpu_util import dev_tensor

pytestmark = pytest.mark.gpu


class Run:
    """A library state of 100,000 parameters and two workers, and moments in `bits` bits."""

    def __init__(self, bits=32, **options):
        hp.hpsgd_destroy()
        hp.hpsgd_init(100_000, 2, 0.1, 0.0, 7)
        for name, value in options.items():
            hp.hpsgd_set_option(getattr(hp, "HPSGD_OPT_" + name), value)
        self.P_pad = hp.hpsgd_get_sizes()[1]
        dt = torch.float32 if bits == 32 else torch.uint8
        self.g = torch.full((self.P_pad,), 1e-3, device="cuda")
        self.m, self.v = (torch.zeros(self.P_pad + 8, dtype=dt, device="cuda") for _ in range(2))
        self.s = [torch.zeros(-(-self.P_pad // 128), dtype=torch.uint8, device="cuda") if bits == 8 else None for _ in range(2)]
        self.bits = bits
        torch.cuda.synchronize()

    def step(self, worker=0, step=1, **change):
        kw = dict(m=self.m, v=self.v, step=step, lr=0.01, state_bits=self.bits, m_scale=self.s[0], v_scale=self.s[1])
        hp.hpsgd_local_step_adamw(worker, change.pop("grads", self.g), **{**kw, **change})

    def __enter__(self):
        return self

    def __exit__(self, *_):
        hp.hpsgd_destroy()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("chunks,fuse", [(1, 0), (3, 0), (1, 2)])
def test_profile_counts_its_launches(bits, chunks, fuse):
    with Run(bits, CHUNKS=chunks, FUSE=fuse, PROFILE=1) as run:
        hp.hpsgd_profile_read(hp.HPSGD_KERNEL_LOCAL_STEP)
        before = hp.hpsgd_launch_count()
        run.step(0)
        run.step(1)
        run.step(0, 2)
        launches = hp.hpsgd_launch_count() - before
        ms, n = hp.hpsgd_profile_read(hp.HPSGD_KERNEL_LOCAL_STEP)
        assert n == launches == 3 * chunks
        assert 0.0 < ms < 1000.0
        hp.hpsgd_set_option(hp.HPSGD_OPT_PROFILE, 0)
        run.step(1, 2)
        assert hp.hpsgd_profile_read(hp.HPSGD_KERNEL_LOCAL_STEP)[1] == 0


@pytest.mark.parametrize("name", ["m", "v", "grad_scale"])
def test_an_unaligned_address_is_refused_before_anything_is_enqueued(name):
    """A held-back local step stays held back: the merge that comes next still runs with it as one kernel."""
    with Run(32, FUSE=2) as run:
        for worker in range(2):
            hp.hpsgd_local_step(worker, run.g)
        before = hp.hpsgd_launch_count()
        with pytest.raises(hp.HpsgdError) as err:
            run.step(0, **{name: run.m.data_ptr() + 2})
        assert err.value.code == hp.HPSGD_E_BADARG
        assert hp.hpsgd_launch_count() == before
        hp.hpsgd_sync_merge()
        assert hp.hpsgd_launch_count() == before + 1
        hp.hpsgd_synchronize()
        assert float(dev_tensor(hp.hpsgd_get_global(), run.P_pad).abs().max()) < 1.0


def test_tensors_that_cannot_be_moments_are_refused():
    with Run(8) as run:
        before = hp.hpsgd_launch_count()
        for change in (dict(m=run.m.cpu()), dict(grads=run.g.cpu()), dict(grad_scale=torch.ones(1)), dict(v=run.v[9:]), dict(m=run.m.float()),
                       dict(m_scale=run.s[0][1:]), dict(v_scale=run.s[1].float()), dict(state_bits=32)):
            with pytest.raises(hp.HpsgdError) as err:
                run.step(0, **change)
            assert err.value.code == hp.HPSGD_E_BADARG
        assert hp.hpsgd_launch_count() == before
        run.step(0)
