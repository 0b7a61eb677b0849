"""hpsgd_adamw_step and hpsgd_grad_norm against their definitions in binary64."""
import math

import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import ops_ref as ref

pytestmark = pytest.mark.gpu

F8, U8, BF, F32 = torch.float8_e4m3fn, torch.uint8, torch.bfloat16, torch.float32
KIND = {F32: hp.HPSGD_F32, BF: hp.HPSGD_BF16}
HY = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=7)
EPS32 = 2.0 ** -24
BIG = 1 << 33        # a position whose upper half is not zero


def up(n, a):
    return -(-n // a) * a


class Tensors:
    """Tensors of the given sizes, each in memory of its own with guard elements around it, `skew` elements off a 256-byte boundary."""

    def __init__(self, sizes, param=F32, grad=F32, bits=32, copy=False, skew=0, seed=0, decay=0.01, rng0=0):
        r = np.random.default_rng(seed)
        self.sizes, self.bits, self.param, self.rows, self.host, self.guards = sizes, bits, param, [], [], []
        at = rng0
        for n in sizes:
            p = self.place(torch.from_numpy(r.normal(size=n, scale=0.05).astype(np.float32)).to(param), skew)
            gv = r.normal(size=n, scale=1e-3) * np.exp(r.normal(size=n)) * (r.random(n) > 0.2)
            g = self.place(torch.from_numpy(gv.astype(np.float32)).to(grad), skew)
            row = {"param": p, "grad": g, "n": n, "rng_offset": at, "weight_decay": decay}
            mv = (r.normal(size=n, scale=3e-4)).astype(np.float32)
            vv = np.square(r.normal(size=n, scale=1e-3)).astype(np.float32)
            nb = -(-n // 128)
            if bits == 32:
                row["m"], row["v"] = self.place(torch.from_numpy(mv), skew), self.place(torch.from_numpy(vv), skew)
                m64, v64 = mv.astype(np.float64), vv.astype(np.float64)
            else:
                for name, x in (("m", mv), ("v", np.sqrt(vv))):
                    q, e = ref.quantize(x.reshape(1, -1))
                    row[name] = self.place(torch.from_numpy(q.reshape(-1)), skew)
                    row[name + "_scale"] = self.place(torch.from_numpy(e.reshape(-1)[:nb].astype(np.uint8)), skew)
                m64, v64 = self.moments(row)
            if copy:
                row["copy"] = self.place(torch.zeros(n, dtype=BF), skew)
            self.host.append({"p": p.double().cpu().numpy(), "g": g.double().cpu().numpy(), "m": m64, "v": v64,
                              "q": at + np.arange(n), "decay": decay})
            self.rows.append(row)
            at += n
        self.table = hp.make_adamw_table(self.rows, KIND[param], KIND[grad], bits)

    def place(self, x, skew):
        pad = 256 // x.element_size()
        buf = torch.full((up(len(x) + skew, pad) + 3 * pad,), 7, dtype=x.dtype, device="cuda")
        view = buf[pad + skew: pad + skew + len(x)]
        view.copy_(x)
        self.guards.append((buf, pad + skew, len(x)))
        return view

    def moments(self, row):
        m = ref.E4M3[row["m"].cpu().numpy()] * np.repeat(ref.factor(row["m_scale"].cpu().numpy()), 128)[: row["m"].numel()]
        r = ref.E4M3[row["v"].cpu().numpy()] * np.repeat(ref.factor(row["v_scale"].cpu().numpy()), 128)[: row["v"].numel()]
        return m, r * r

    def guards_hold(self):
        for buf, at, n in self.guards:
            assert bool((buf[:at] == 7).all()) and bool((buf[at + n:] == 7).all())


def check(t, seed, c=1.0, hy=HY):
    """The tensors after one step against binary64.  Bounds: a handful of binary32 roundings on the terms' magnitudes for what is
    kept in 32 bits; for codes the same neighbour, unless the draw is so near to the turning point that binary32 can tip it (x is known to
    about 8 roundings, 16 codes to an octave: 8 * 16 * 2^-24 of a step, 3e-5 allows four times that)."""
    for row, h, n in zip(t.rows, t.host, t.sizes):
        p, m, v = ref.adamw(h["p"], h["g"], h["m"], h["v"], hy["lr"], hy["beta1"], hy["beta2"], hy["eps"], hy["step"], h["decay"], c)
        mag = hy["lr"] * np.abs(m) / (1 - hy["beta1"] ** hy["step"]) / (np.sqrt(v / (1 - hy["beta2"] ** hy["step"])) + hy["eps"])
        # cancellation in m: its terms, not its value, bound its error
        terms = np.abs(hy["beta1"] * h["m"]) + np.abs((1 - hy["beta1"]) * h["g"] * c)
        ratio = np.divide(terms, np.abs(m), out=np.ones_like(m), where=m != 0)
        tol_p = EPS32 * (3 * np.abs(h["p"]) + mag * (12 + 4 * ratio)) + 1e-30
        got = row["param"].double().cpu().numpy()
        if t.param == F32:
            assert np.all(np.abs(got - p) <= tol_p), np.max(np.abs(got - p) / tol_p)
            if "copy" in row:
                assert torch.equal(row["copy"], row["param"].to(BF))
        else:
            rnd = ref.random_bits(seed, hy["step"], h["q"])
            ulp = np.ldexp(1.0, np.frexp(np.maximum(np.abs(p), 2.0 ** -126))[1] - 8)
            s = np.abs(p) / ulp + ((rnd * ref.N2 & 0xFFFFFFFF) >> 16) / 65536.0
            want = np.sign(p) * np.floor(s) * ulp
            near = np.abs(s - np.round(s)) * ulp <= tol_p * 2
            assert np.all((got == want) | (near & (np.abs(got - want) <= ulp * 1.001))), "bf16 rounding"
        if t.bits == 32:
            assert np.all(np.abs(row["m"].double().cpu().numpy() - m) <= 4 * EPS32 * terms + 1e-44)
            assert np.all(np.abs(row["v"].double().cpu().numpy() - v) <= 8 * EPS32 * v + 1e-44)
            continue
        rnd = ref.random_bits(seed, hy["step"], h["q"])
        for name, x, rounded, r16 in (("m", m, ref.round_first, rnd >> 16), ("v", np.sqrt(v), ref.round_second, rnd & 0xFFFF)):
            top = np.abs(ref.blocks(x.reshape(1, -1))[0]).max(axis=1)
            e = ref.scale_bytes(top)
            got_e = row[name + "_scale"].cpu().numpy().astype(np.int64)
            edge = np.abs(top / (448 * ref.factor(np.minimum(e, got_e))) - 1) < 1e-6
            assert np.all((e == got_e) | edge)
            f = np.repeat(ref.factor(got_e), 128)[:n]
            want, room = rounded(np.clip(x / f, -448, 448), r16)
            got = ref.E4M3[row[name].cpu().numpy()]
            slack = np.where(name == "m", 3e-5 * np.maximum(1.0, terms / np.maximum(np.abs(m), 1e-300)), 3e-5)
            off = got != want
            assert np.all(room[off] <= slack[off]), (name, room[off][:5])
            assert np.all(np.abs(got - want)[off] <= np.maximum(np.abs(want[off]), 2.0 ** -6) / 7.9)
    t.guards_hold()


SIZES = [[1], [7], [8], [127], [128], [129], [1023], [1024], [1025], [3, 1, 128, 2000, 5, 4096, 77], [64] * 11, [20011]]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [(F32, F32), (F32, BF), (BF, F32), (BF, BF)])
def test_one_step(sizes, bits, param, grad):
    t = Tensors(sizes, param, grad, bits, copy=param == F32, seed=sum(sizes))
    hp.hpsgd_adamw_step(t.table, seed=11, **HY)
    check(t, 11)


@pytest.mark.parametrize("skew", [1, 3, 4])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", [F32, BF])
def test_tensors_off_any_wide_boundary(skew, bits, param):
    t = Tensors([1000, 129, 5], param, BF, bits, copy=param == F32, skew=skew, seed=skew)
    hp.hpsgd_adamw_step(t.table, seed=5, **HY)
    check(t, 5)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_one_launch_takes_and_empty_ones(bits):
    sizes = [1 + (37 * k) % 300 for k in range(801)]
    t = Tensors(sizes, F32, F32, bits, seed=1)
    rows = []
    for k, row in enumerate(t.rows):
        rows.append(row)
        if k % 100 == 0:
            rows.append({"n": 0, "rng_offset": row["rng_offset"] + row["n"]})
    table = hp.make_adamw_table(rows, hp.HPSGD_F32, hp.HPSGD_F32, bits)
    hp.hpsgd_adamw_step(table, seed=3, **HY)
    check(t, 3)


@pytest.mark.parametrize("param", [F32, BF])
def test_random_positions_beyond_32_bits(param):
    t = Tensors([300], param, F32, 8, rng0=BIG - 100, seed=2)      # the position's upper half changes inside the tensor
    hp.hpsgd_adamw_step(t.table, seed=1 << 63, **HY)
    check(t, 1 << 63)


@pytest.mark.parametrize("hy", [dict(HY, step=1), dict(HY, beta1=0.0, beta2=0.0), dict(HY, lr=0.0), dict(HY, eps=1e-3, step=10 ** 9),
                                dict(HY, beta2=0.95, lr=0.1)], ids=str)
@pytest.mark.parametrize("bits", [32, 8])
def test_hyperparameters(hy, bits):
    t = Tensors([515, 64], F32, F32, bits, seed=4, decay=0.1)
    hp.hpsgd_adamw_step(t.table, seed=9, **hy)
    check(t, 9, hy=hy)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zero_state(bits):
    """From zero moments the first step is lr * sign(g) wherever |g| is far above eps."""
    n = 1000
    g = torch.randn(n, device="cuda")
    p = torch.zeros(n, device="cuda")
    dt = F32 if bits == 32 else U8
    st = {k: torch.zeros(n, dtype=dt, device="cuda") for k in "mv"}
    sc = {k + "_scale": torch.zeros(8, dtype=U8, device="cuda") for k in "mv"} if bits == 8 else {}
    t = hp.make_adamw_table([dict(param=p, grad=g, n=n, **st, **sc)], hp.HPSGD_F32, hp.HPSGD_F32, bits)
    hp.hpsgd_adamw_step(t, 0.01, 0.9, 0.999, 1e-12, 1)
    assert torch.allclose(p, -0.01 * g.sign(), rtol=1e-5, atol=0)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradient_scale_and_skipped_step(bits):
    t = Tensors([700, 128], F32, BF, bits, seed=6)
    hp.hpsgd_adamw_step(t.table, seed=2, grad_scale=torch.tensor([0.25], device="cuda"), **HY)
    check(t, 2, c=0.25)
    before = [buf.clone() for buf, _, _ in t.guards]
    for bad in (math.nan, math.inf, -math.inf):
        hp.hpsgd_adamw_step(t.table, seed=2, grad_scale=torch.tensor([bad], device="cuda"), **HY)
    assert all(torch.equal(a, b[0]) for a, b in zip(before, t.guards))


def test_infinite_and_nan_gradients_stay_in_their_elements():
    """8-bit moments: an element that is not finite gets the NaN code and does not touch its block's scale or neighbours."""
    a, b = Tensors([384], F32, F32, 8, seed=8), Tensors([384], F32, F32, 8, seed=8)
    bad = [5, 130, 383]
    a.rows[0]["grad"][bad] = torch.tensor([math.inf, -math.inf, math.nan], device="cuda")
    b.rows[0]["grad"][bad] = 0.0
    b.rows[0]["m"][bad] = 0        # nor do they count in the comparison
    b.rows[0]["v"][bad] = 0
    for t in (a, b):
        hp.hpsgd_adamw_step(t.table, seed=1, **HY)
    keep = torch.ones(384, dtype=torch.bool)
    keep[bad] = False
    for name in ("param", "m", "v", "m_scale", "v_scale"):
        x, y = a.rows[0][name].cpu(), b.rows[0][name].cpu()
        assert torch.equal(x, y) if "scale" in name else torch.equal(x[keep], y[keep]), name
    assert a.rows[0]["m"].cpu()[bad].tolist() == [0x7F] * 3 and a.rows[0]["v"].cpu()[bad].tolist() == [0x7F] * 3
    assert not torch.isfinite(a.rows[0]["param"].cpu()[bad]).any()


def test_bf16_parameters_that_are_not_finite_stay_so():
    n = 256
    p = torch.zeros(n, dtype=torch.int16, device="cuda").view(BF)
    p.view(torch.int16)[:4] = torch.tensor([0x7F80, -0x80, 0x7FFF, -1], dtype=torch.int16, device="cuda")     # inf, -inf, NaN, NaN
    z = lambda: torch.zeros(n, device="cuda")  # noqa: E731
    t = hp.make_adamw_table([dict(param=p, grad=z(), m=z(), v=z(), n=n)], hp.HPSGD_BF16, hp.HPSGD_F32, 32)
    hp.hpsgd_adamw_step(t, seed=3, **HY)
    x = p.float().cpu()
    assert x[0] == math.inf and x[1] == -math.inf and math.isnan(x[2]) and math.isnan(x[3]) and bool((x[4:] == 0).all())


def test_rounding_keeps_expected_values():
    """Over many draws the mean of m and the mean of r^2 are the unrounded moments: within 5 standard errors."""
    n, draws = 4096, 400
    t = Tensors([n], F32, F32, 8, seed=12)
    h = t.host[0]
    start = {k: t.rows[0][k].clone() for k in ("m", "v", "m_scale", "v_scale")}
    sums = np.zeros((2, n))
    squares = np.zeros((2, n))
    for s in range(draws):
        for k, x in start.items():
            t.rows[0][k].copy_(x)
        hp.hpsgd_adamw_step(t.table, seed=s, **HY)
        mv = np.stack(t.moments(t.rows[0]))
        sums += mv
        squares += mv * mv
    _, m, v = ref.adamw(h["p"], h["g"], h["m"], h["v"], HY["lr"], 0.9, 0.999, HY["eps"], 7, 0.0)
    low = np.repeat(ref.factor(t.rows[0]["v_scale"].cpu().numpy()), 128)[:n] * 2.0 ** -9
    for k, want, use in ((0, m, np.ones(n, bool)), (1, v, np.sqrt(v) > low)):
        mean = sums[k] / draws
        var = np.maximum(squares[k] / draws - mean ** 2, 0)
        z = ((mean - want) / np.sqrt(var / draws + 1e-40))[use & (var > 0)]
        # z of a mean over 400 draws of two values has heavy tails where one of them is rare: the average over elements is what is tested
        assert abs(z.mean()) < 5 / math.sqrt(len(z)) + 0.02 and 0.8 < z.std() < 1.3


def test_second_moment_decays_without_gradient():
    """A thousand steps without gradient: v falls by 0.999^1000.  Rounded to nearest it would stay where it is."""
    n, steps = 16384, 1000
    t = Tensors([n], F32, F32, 8, seed=13, decay=0.0)
    t.rows[0]["grad"].zero_()
    _, v0 = t.moments(t.rows[0])
    for s in range(steps):
        hp.hpsgd_adamw_step(t.table, 0.0, 0.9, 0.999, 1e-8, s + 1, seed=1)
    _, v1 = t.moments(t.rows[0])
    use = v0 > 1e-3 * v0.max()
    assert abs(v1[use].sum() / v0[use].sum() / 0.999 ** steps - 1) < 0.02


def test_descends_as_in_32_bits():
    """A least-squares problem: 8-bit moments reach the loss that 32-bit moments reach, within a factor of 1.5."""
    torch.manual_seed(0)
    n = 2048
    A = torch.randn(n, n, device="cuda") / math.sqrt(n)
    y = torch.randn(n, device="cuda")
    loss = {}
    for bits in (32, 8):
        p = torch.zeros(n, device="cuda")
        g = torch.zeros(n, device="cuda")
        dt = F32 if bits == 32 else U8
        row = dict(param=p, grad=g, m=torch.zeros(n, dtype=dt, device="cuda"), v=torch.zeros(n, dtype=dt, device="cuda"), n=n)
        if bits == 8:
            row |= dict(m_scale=torch.zeros(16, dtype=U8, device="cuda"), v_scale=torch.zeros(16, dtype=U8, device="cuda"))
        t = hp.make_adamw_table([row], hp.HPSGD_F32, hp.HPSGD_F32, bits)
        for s in range(300):
            e = A @ p - y
            g.copy_(A.t() @ e)
            hp.hpsgd_adamw_step(t, 0.02, 0.9, 0.99, 1e-8, s + 1, seed=4)
        loss[bits] = float((A @ p - y).square().mean())
    assert loss[8] < 1.5 * loss[32] < 0.5 * float(y.square().mean())


def test_a_captured_step_replays():
    t, u = (Tensors([5000, 3], F32, F32, 8, seed=14) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    ws, out = torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8, device="cuda"), torch.zeros(2, device="cuda")
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        hp.hpsgd_grad_norm(t.table, 0.01, ws, out, stream=s)
        hp.hpsgd_adamw_step(t.table, seed=1, grad_scale=out[1:], stream=s, **HY)
    for _ in range(3):
        graph.replay()
        hp.hpsgd_grad_norm(u.table, 0.01, ws, out)
        hp.hpsgd_adamw_step(u.table, seed=1, grad_scale=out[1:], **HY)
    for a, b in zip(t.guards, u.guards):
        assert torch.equal(a[0], b[0])


# ---------------------------------------------------------------------------------------------- the norm
@pytest.mark.parametrize("sizes", [[], [1], [0, 5], [8192], [8193, 1, 0, 7], [3_000_001, 12345], [50] * 900], ids=lambda s: str(s)[:20])
@pytest.mark.parametrize("grad", [F32, BF])
@pytest.mark.parametrize("skew", [0, 1])
def test_norm(sizes, grad, skew):
    r = np.random.default_rng(len(sizes))
    rows, total = [], 0.0
    for n in sizes:
        buf = torch.full((n + 64,), 9.0, device="cuda").to(grad)
        x = buf[skew: skew + n]
        x.copy_(torch.from_numpy(r.normal(size=n).astype(np.float32)))
        total += float(x.double().square().sum())
        rows.append({"grad": x, "n": n})
    ws = torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8, device="cuda")
    out = torch.full((2,), 5.0, device="cuda")
    table = hp.make_adamw_table(rows, hp.HPSGD_F32, KIND[grad], 32)
    norm = math.sqrt(total)
    got = []
    for most in (0.5, 1e9, math.inf):
        hp.hpsgd_grad_norm(table, most, ws, out)
        a, c = out.cpu().tolist()
        got.append(a)
        # squares in groups of eight: at most 8 roundings, halved by the root, and the rounding of the result
        assert abs(a - norm) <= 5 * EPS32 * norm
        want = most / norm if norm > most else 1.0
        assert abs(c - want) <= 6 * EPS32 * want
    assert len(set(got)) == 1


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan, 3e38])
def test_norm_that_is_not_finite(bad):
    x = torch.ones(5000, device="cuda")
    x[4321] = bad
    x[17] = bad
    ws, out = torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8, device="cuda"), torch.zeros(2, device="cuda")
    hp.hpsgd_grad_norm(hp.make_adamw_table([{"grad": x, "n": 5000}], 0, 0, 32), 1.0, ws, out)
    a, c = out.cpu().tolist()
    assert not math.isfinite(a) and math.isnan(c)


def test_work_is_ordered_on_the_stream_it_is_given():
    side = torch.cuda.Stream()
    n = 1 << 22
    x = torch.zeros(n, device="cuda")
    ws, out = torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8, device="cuda"), torch.zeros(2, device="cuda")
    table = hp.make_adamw_table([{"grad": x, "n": n}], 0, 0, 32)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for k in range(20):
            x.fill_(float(k))
            hp.hpsgd_grad_norm(table, 1.0, ws, out, stream=side)
    side.synchronize()
    assert out[0].item() == 19.0 * 2048.0
