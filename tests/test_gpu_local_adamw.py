"""hpsgd_local_step_adamw: the AdamW operator on a worker's replica under every schedule, and a few of its refusals."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests.gpu_util import dev_tensor

pytestmark = pytest.mark.gpu

SIZES, K, SEED, LR = [1000, 77, 40_000], 3, 21, 1e-2
M1 = 0x6A09E667F3BCC909


class Moments:
    def __init__(self, n, bits):
        self.bits = bits
        dt = torch.float32 if bits == 32 else torch.uint8
        self.m, self.v = (torch.zeros(n, dtype=dt, device="cuda") for _ in range(2))
        nb = -(-n // 128)
        self.s = [torch.zeros(nb, dtype=torch.uint8, device="cuda") for _ in range(2)] if bits == 8 else [None, None]


def gradients(P_pad, offsets, dtype):
    """[round][step][worker]; zeros in the pads."""
    g = torch.Generator(device="cuda").manual_seed(5)
    live = torch.zeros(P_pad, device="cuda")
    for n, o in zip(SIZES, offsets):
        live[o:o + n] = 1.0
    return [[[(torch.randn(P_pad, generator=g, device="cuda") * live * 1e-3).to(dtype) for _ in range(K)] for _ in range(2)] for _ in range(4)]


def steps_of(t, i):
    """Local steps of worker i in round t: one, but two or none here and there."""
    return {(1, 0): 2, (2, 2): 0}.get((t, i), 1)


def expected(w, grads, bits, dtype, staleness):
    """The same rounds by the operator on separate replicas and a merge in numpy's binary32."""
    P_pad = w.size
    mom, count = [Moments(P_pad, bits) for _ in range(K)], [0] * K
    D, first = np.zeros_like(w), True
    for t in range(4):
        rows = []
        for i in range(K):
            r = torch.from_numpy(w.copy()).cuda()
            for s in range(steps_of(t, i)):
                count[i] += 1
                table = hp.make_adamw_table([dict(param=r, grad=grads[t][s][i], m=mom[i].m, v=mom[i].v, m_scale=mom[i].s[0], v_scale=mom[i].s[1],
                                                  n=P_pad, weight_decay=0.1)], hp.HPSGD_F32, dtype, bits)
                hp.hpsgd_adamw_step(table, LR, 0.9, 0.99, 1e-8, count[i], (SEED + i * M1) % 2 ** 64)
            rows.append(r.cpu().numpy())
        acc = rows[0] - w
        for r in rows[1:]:
            acc = acc + (r - w)
        new = acc / np.float32(K)
        if staleness == 0:
            w = w + new
        elif not first:
            w = w + D
        D, first = new, False
    return w


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [hp.HPSGD_F32, hp.HPSGD_BF16])
@pytest.mark.parametrize("schedule", [dict(), dict(chunks=3), dict(overlap=0), dict(fuse=1), dict(fuse=2), dict(fuse=2, chunks=2), dict(pipeline=1),
                                      dict(staleness=0)], ids=str)
def test_rounds(bits, dtype, schedule):
    hp.hpsgd_destroy()
    hp.hpsgd_set_layout(SIZES)
    P_pad, offsets = hp.hpsgd_layout_padded(SIZES)
    hp.hpsgd_set_pipeline(schedule.get("pipeline", 0))
    hp.hpsgd_init(sum(SIZES), K, 0.1, 0.0, SEED)
    try:
        for key, name in ((hp.HPSGD_OPT_CHUNKS, "chunks"), (hp.HPSGD_OPT_OVERLAP, "overlap"), (hp.HPSGD_OPT_FUSE, "fuse"), (hp.HPSGD_OPT_STALENESS, "staleness")):
            if name in schedule:
                hp.hpsgd_set_option(key, schedule[name])
        hp.hpsgd_set_option(hp.HPSGD_OPT_GRAD_DTYPE, dtype)
        w0 = dev_tensor(hp.hpsgd_get_global(), P_pad).cpu().numpy().copy()
        grads = gradients(P_pad, offsets, torch.float32 if dtype == hp.HPSGD_F32 else torch.bfloat16)
        torch.cuda.synchronize()
        mom, count = [Moments(P_pad, bits) for _ in range(K)], [0] * K
        torch.cuda.synchronize()          # the library works on streams of its own
        before = hp.hpsgd_launch_count()
        for t in range(4):
            for i in range(K):
                for s in range(steps_of(t, i)):
                    count[i] += 1
                    hp.hpsgd_local_step_adamw(i, grads[t][s][i], mom[i].m, mom[i].v, count[i], LR, 0.9, 0.99, 1e-8, 0.1, bits, mom[i].s[0], mom[i].s[1])
            hp.hpsgd_sync_merge()
        got = dev_tensor(hp.hpsgd_get_global(), P_pad).cpu().numpy().copy()
        assert hp.hpsgd_launch_count() > before
    finally:
        hp.hpsgd_destroy()
    want = expected(w0, grads, bits, dtype, schedule.get("staleness", 1))
    assert np.array_equal(got.view(np.int32), want.view(np.int32))
    assert not np.array_equal(got, w0)


def test_mixed_with_sgd_steps_and_a_gradient_scale():
    """An SGD step (held back by HPSGD_OPT_FUSE 2) and an AdamW step of the same round happen in their order; a scale that is not finite skips."""
    P = 5000
    hp.hpsgd_destroy()
    hp.hpsgd_init(P, 1, 0.5, 0.0, 3)
    try:
        hp.hpsgd_set_option(hp.HPSGD_OPT_FUSE, 2)
        hp.hpsgd_set_option(hp.HPSGD_OPT_STALENESS, 0)
        P_pad = hp.hpsgd_get_sizes()[1]
        w = dev_tensor(hp.hpsgd_get_global(), P_pad).clone()
        g = torch.zeros(P_pad, device="cuda")
        g[:P] = 1.0
        mo, bad = Moments(P_pad, 32), torch.tensor([float("nan")], device="cuda")
        torch.cuda.synchronize()
        hp.hpsgd_local_step(0, g)
        hp.hpsgd_local_step_adamw(0, g, mo.m, mo.v, 1, 0.25, grad_scale=bad)
        hp.hpsgd_local_step_adamw(0, g, mo.m, mo.v, 1, 0.25)
        hp.hpsgd_sync_merge()
        hp.hpsgd_synchronize()
        got = dev_tensor(hp.hpsgd_get_global(), P_pad)[:P]
        # SGD: -0.5; the first AdamW step: -0.25 * 1 / (1 + eps), each within a few roundings of numbers below 1
        assert float((got - (w[:P] - 0.75)).abs().max()) < 1e-6
    finally:
        hp.hpsgd_destroy()


def test_refusals():
    hp.hpsgd_destroy()
    hp.hpsgd_init(1000, 2, 0.1, 0.0, 1)
    try:
        g = torch.zeros(1024, device="cuda")
        mo = Moments(1024, 8)
        torch.cuda.synchronize()
        ok = dict(m=mo.m, v=mo.v, step=1, lr=0.1, state_bits=8, m_scale=mo.s[0], v_scale=mo.s[1])
        for worker, grads, change in ((2, g, {}), (0, None, {}), (0, g, dict(m=None)), (0, g, dict(v_scale=None)), (0, g, dict(step=0)), (0, g, dict(lr=-1.0)),
                                      (0, g, dict(beta2=1.0)), (0, g, dict(state_bits=4)), (0, g, dict(weight_decay=-1.0))):
            with pytest.raises(hp.HpsgdError) as err:
                hp.hpsgd_local_step_adamw(worker, grads, **{**ok, **change})
            assert err.value.code == hp.HPSGD_E_BADARG
        hp.hpsgd_local_step_adamw(1, g, **ok)
        hp.hpsgd_synchronize()
    finally:
        hp.hpsgd_destroy()
    with pytest.raises(hp.HpsgdError) as err:
        hp.hpsgd_local_step_adamw(0, g, **ok)
    assert err.value.code == hp.HPSGD_E_STATE
    hp.hpsgd_set_form(hp.HPSGD_FORM_GRADIENT_ACCUMULATION)
    hp.hpsgd_init(1000, 2, 0.1, 0.0, 1)
    try:
        with pytest.raises(hp.HpsgdError) as err:
            hp.hpsgd_local_step_adamw(0, g, **ok)
        assert err.value.code == hp.HPSGD_E_STATE
    finally:
        hp.hpsgd_destroy()
