"""hpsgd_adamw_step with 8-bit moments where a block's second moments lie many octaves apart, are zero, very large or not
finite: code by code against the definition in binary64."""
import math

import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import ops_ref as ref
from tests.test_gpu_adamw import BF, EPS32, F32, HY, KIND, U8, Tensors, check

pytestmark = pytest.mark.gpu


def ladder(lo, hi, n=128):
    return np.float32(10.0) ** np.linspace(lo, hi, n).astype(np.float32)


# Gradients of one block each, from zero moments.  With beta2 = 0.999 the second moment is g^2 / 1000: from 1e-43 (a subnormal number, still
# positive) up.
BLOCKS = {
    "from 1e-20 to 1": ladder(-20, 0),
    "zeros": np.zeros(128, np.float32),
    "every other one zero": np.where(np.arange(128) % 2, 0.3, 0.0) * ladder(-3, 0),
    "one far above the rest": np.concatenate([np.full(127, 1e-9), [3e4]]),
    "one zero": np.concatenate([ladder(-4, -1, 127), [0.0]]),
    "a tenth zero": np.where(np.arange(128) % 10 == 3, 0.0, 1e-3) * ladder(0, 1),
    "all tiny": np.full(128, 1e-18, np.float32),
    "beyond 448 * 2^6": ladder(2, 8),
    "beyond 448 * 2^6, and tiny ones": np.concatenate([ladder(4, 9, 64), ladder(-19, -12, 64)]),
    "ordinary": 1e-3 * np.abs(np.random.default_rng(3).normal(size=128)),
}


def gradients(n, signs):
    g = np.resize(np.concatenate(list(BLOCKS.values())), n).astype(np.float32)
    return np.where(signs, -g, g).astype(np.float32)


def with_gradients(n, param, grad, skew, seed):
    """Tensors from zero moments with the blocks above as gradients, again and again."""
    t = Tensors([n], param, grad, 8, skew=skew, seed=seed)
    row, host = t.rows[0], t.host[0]
    row["grad"].copy_(torch.from_numpy(gradients(n, np.random.default_rng(seed).random(n) < 0.5)))
    for name in ("m", "v", "m_scale", "v_scale"):
        row[name].zero_()
    host["g"], host["m"], host["v"] = row["grad"].double().cpu().numpy(), np.zeros(n), np.zeros(n)
    return t


# 2085 elements end in a part of a block; two chunks of 1024 take the wide form, the rest and the skewed ones the other.
@pytest.mark.parametrize("n,skew", [(2085, 0), (2560, 0), (1280, 3)])
@pytest.mark.parametrize("param,grad", [(F32, F32), (F32, BF), (BF, BF)])
def test_blocks_of_every_spread(n, skew, param, grad):
    for seed in range(3):
        t = with_gradients(n, param, grad, skew, seed)
        hp.hpsgd_adamw_step(t.table, seed=seed, **HY)
        check(t, seed)
        # the rule by itself: a positive second moment has a positive code, a zero one has none
        positive = torch.from_numpy(t.host[0]["g"]).abs() > 0
        code = t.rows[0]["v"].cpu()
        assert bool(((code > 0) == positive).all())


def test_an_old_spike_does_not_erase_its_neighbours():
    """A gradient 10^13 times its neighbours', then none: the neighbours keep a second moment, so their next step divides by it and not by
    eps alone."""
    n, eps = 128, 1e-30
    g = torch.full((n,), 1e-9, device="cuda")
    g[77] = 1e4
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=U8, device="cuda"), torch.zeros(n, dtype=U8, device="cuda")
    s = [torch.zeros(1, dtype=U8, device="cuda") for _ in range(2)]
    row = dict(param=p, grad=g, m=m, v=v, m_scale=s[0], v_scale=s[1], n=n)
    table = hp.make_adamw_table([row], hp.HPSGD_F32, hp.HPSGD_F32, 8)
    hp.hpsgd_adamw_step(table, 1e-3, 0.9, 0.999, eps, 1, seed=5)
    assert bool((v > 0).all())
    # the next step with a first moment of the neighbours' own size in a block of its own scale
    q, e = ref.quantize(np.full((1, n), 1e-10))
    m.copy_(torch.from_numpy(q.reshape(-1)))
    s[0].copy_(torch.from_numpy(e.reshape(-1).astype(np.uint8)))
    g.zero_()
    p.zero_()
    r = ref.E4M3[v.cpu().numpy()] * ref.factor(s[1].cpu().numpy())[0]
    m64 = ref.E4M3[q.reshape(-1)] * ref.factor(e)[0, 0]
    hp.hpsgd_adamw_step(table, 1e-3, 0.9, 0.999, eps, 2, seed=5)
    want, _, _ = ref.adamw(0.0, 0.0, m64, r * r, 1e-3, 0.9, 0.999, eps, 2, 0.0)
    # a product, a root, a sum, a reciprocal (one unit in the last place), two products: 12 roundings of binary32 are more than there are
    assert np.all(np.abs(p.double().cpu().numpy() - want) <= 12 * EPS32 * np.abs(want))
    assert float(p.abs().max()) < 1.0


def test_blocks_that_are_not_finite_keep_the_rule():
    """Infinity and NaN beside second moments of every size: they count for no scale, and the positive ones stay positive."""
    n = 1280
    t, u = (with_gradients(n, F32, F32, 0, 9) for _ in range(2))
    bad = [3, 200, 400, 600, 1000, 1279]
    t.rows[0]["grad"][bad] = torch.tensor([math.inf, -math.inf, math.nan, math.inf, math.nan, -math.inf], device="cuda")
    u.rows[0]["grad"][bad] = 0.0
    u.host[0]["g"][bad] = 0.0
    for x in (t, u):
        hp.hpsgd_adamw_step(x.table, seed=2, **HY)
    check(u, 2)
    keep = torch.ones(n, dtype=torch.bool)
    keep[bad] = False
    for name in ("param", "m", "v"):
        assert torch.equal(t.rows[0][name].cpu()[keep], u.rows[0][name].cpu()[keep]), name
    for name in ("m_scale", "v_scale"):
        assert torch.equal(t.rows[0][name], u.rows[0][name])
    assert t.rows[0]["v"].cpu()[bad].tolist() == [0x7F] * len(bad)


@pytest.mark.parametrize("param,grad", [(F32, F32), (BF, BF)])
def test_blocks_of_two_chunks_give_the_codes_of_one(param, grad):
    """From 4.85 M elements a block takes two chunks of 1024; the same tensors in four calls take one, whose codes the tests against
    binary64 cover: every bit has to be the same."""
    sizes = [5_000_000 + 37, 3000, 1, 777_777]
    assert sum(sizes) >= 2 * 1024 * 148 * 16
    r = torch.Generator(device="cuda").manual_seed(4)
    both, base = [], {}
    for n in sizes:
        size = torch.exp(2 * torch.randn(-(-n // 64), generator=r, device="cuda")).repeat_interleave(64)[:n]
        empty = torch.rand(n, generator=r, device="cuda") < 0.05
        base[n] = (torch.randn(n, generator=r, device="cuda").mul(0.05).to(param), (torch.randn(n, generator=r, device="cuda") * 1e-3 * size * ~empty).to(grad))
    for pieces in (1, 4):
        rows, parts, at = [], [], 0
        for n in sizes:
            nb = -(-n // 128)
            x = dict(param=base[n][0].clone(), grad=base[n][1].clone(), m=torch.zeros(n, dtype=U8, device="cuda"), v=torch.zeros(n, dtype=U8, device="cuda"),
                     m_scale=torch.zeros(nb, dtype=U8, device="cuda"), v_scale=torch.zeros(nb, dtype=U8, device="cuda"))
            rows.append(x)
            cut = -(-n // pieces // 1024) * 1024 if pieces > 1 else n
            for lo in range(0, n, cut):
                hi = min(n, lo + cut)
                parts.append({k: y[lo // 128:] if "scale" in k else y[lo:hi] for k, y in x.items()} | dict(n=hi - lo, rng_offset=at + lo, weight_decay=0.01))
            at += n
        # the large call in one table; the small ones a piece at a time
        for call in ([parts] if pieces == 1 else [[x] for x in parts]):
            table = hp.make_adamw_table(call, KIND[param], KIND[grad], 8)
            for step in (1, 2):
                hp.hpsgd_adamw_step(table, 1e-3, 0.9, 0.999, 1e-8, step, seed=6)
        both.append(rows)
    for a, b in zip(*both):
        for name in a:
            assert torch.equal(a[name], b[name]), name
