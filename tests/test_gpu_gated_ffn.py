"""hpsgd_gated_ffn_forward / _backward against their definitions in binary64."""
import math

import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import ffn_ref as ref
from tests import ops_ref
from tests.test_gpu_norm import Codes

pytestmark = pytest.mark.gpu

U8, BF, F32 = torch.uint8, torch.bfloat16, torch.float32
KIND = {F32: hp.HPSGD_F32, BF: hp.HPSGD_BF16}
ACT = {"silu": hp.HPSGD_SILU, "gelu": hp.HPSGD_GELU}
E32, E16 = 2.0 ** -24, 2.0 ** -8
MARK = 7.0


def up(n, a):
    return -(-n // a) * a


class Operand:
    """Values in the block format; what the format pads with, and what lies behind it, is filled with NaN codes and the largest scales."""

    def __init__(self, x, ld=0, lds=0):
        rows, cols = x.shape
        q, e = ops_ref.quantize(x)
        self.ld, self.lds, nb = ld or up(cols, 16), lds or rows, e.shape[1]
        codes, s = np.full((rows, self.ld), 0x7F, np.uint8), np.full((up(nb, 4) // 4, self.lds, 4), 0xFE, np.uint8)
        codes[:, :cols] = q
        full = np.full((rows, up(nb, 4)), 0xFE)
        full[:, :nb] = e
        s[:, :rows] = full.reshape(rows, -1, 4).transpose(1, 0, 2)
        self.q, self.s, self.values = torch.from_numpy(codes).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(ops_ref.values(q, e)).cuda()


def codes_within(got, x, err):
    """Codes and scales of numbers that lie within `err` of x: their blocks' tops decide the scale, and a code is the nearest of one of them."""
    q, e = got
    b, d = ops_ref.blocks(np.abs(x)), ops_ref.blocks(err)
    assert np.all(e >= ops_ref.scale_bytes(np.maximum(b - d, 0.0).max(axis=2))) and np.all(e <= ops_ref.scale_bytes((b + d).max(axis=2)))
    f = np.repeat(ops_ref.factor(e), 128, axis=1)[:, : x.shape[1]]
    near = lambda y: ops_ref.E4M3[ops_ref.nearest_code(np.clip(y / f, -448, 448))]  # noqa: E731
    v = ops_ref.E4M3[q]
    assert np.all((v >= near(x - err)) & (v <= near(x + err)))


def inputs(M, N, K, seed, scale=1.0, **kw):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(M, K)) * np.exp(rng.normal(size=K) * 0.5)
    w = rng.normal(size=(2 * N, K)) * (scale / math.sqrt(K))
    return Operand(x, **kw), Operand(w, **kw)


class Forward:
    def __init__(self, M, N, K, act, x, w, z_dtype=F32, ldz=0, ldgu=0, skew=0, ldz8=0, ldsz=0):
        self.M, self.N, self.K, self.kind, self.x, self.w, self.skew = M, N, K, act, x, w, skew
        self.ldz, self.ldgu = ldz or N, ldgu or 2 * N
        self.zbuf = torch.full((M * self.ldz + skew + 32,), MARK, dtype=z_dtype, device="cuda")
        self.gubuf = torch.full((M * self.ldgu + skew + 32,), MARK, dtype=BF, device="cuda")
        self.z, self.gu = self.zbuf[skew: skew + M * self.ldz].view(M, self.ldz)[:, :N], self.gubuf[skew: skew + M * self.ldgu].view(M, self.ldgu)[:, : 2 * N]
        self.z8 = Codes(M, N, ldz8, ldsz)

    def args(self, **change):
        kw = dict(x=self.x.q, x_scale=self.x.s, w=self.w.q, w_scale=self.w.s, z8=self.z8.q, z_scale=self.z8.s, z=self.z, z_dtype=KIND[self.z.dtype], gu=self.gu,
                  ldx=self.x.ld, ldsx=self.x.lds, ldw=self.w.ld, ldsw=self.w.lds, ldz=self.ldz, ldgu=self.ldgu, ldz8=self.z8.ld, ldsz=self.z8.lds)
        return hp.make_gated_ffn_forward(self.M, self.N, self.K, ACT[self.kind], **{**kw, **change})

    def run(self, **change):
        hp.hpsgd_gated_ffn_forward(self.args(**change))
        hp.hpsgd_ops_check()

    def want(self):
        """g, u, z and their bounds.  The sums': as for hpsgd_gemm_fp8 (one unit in the last place of the sum of magnitudes an addition, over K / 4 + 8 of them).
        z: no slope is above 1.13; a product and its rounding."""
        y, mag = self.x.values @ self.w.values.t(), self.x.values.abs() @ self.w.values.abs().t()
        y, tol = y.cpu().numpy(), (2 * E32 * (self.K / 4 + 8) * mag).cpu().numpy()
        g, u, tg, tu = y[:, : self.N], y[:, self.N:], tol[:, : self.N], tol[:, self.N:]
        a = ref.act(g, self.kind)
        ea = ref.act_error(np.abs(g) + tg, self.kind) + ref.act_error(-np.abs(g) - tg, self.kind) + 1.13 * tg
        z = a * u
        return y, tol, z, ea * (np.abs(u) + tu) + np.abs(a) * tu + np.abs(z) * 2 * E32 + 2.0 ** -126

    def check(self):
        y, tol, z, ez = self.want()
        gu = self.gu.double().cpu().numpy()
        assert np.all(np.abs(gu - y) <= tol + E16 * (np.abs(y) + tol))
        got = self.z.double().cpu().numpy()
        off = np.abs(got - z) - ez - (E16 if self.z.dtype == BF else 0.0) * (np.abs(z) + ez)
        assert np.all(off <= 0), (off.max(), np.argwhere(off > 0)[:4])
        codes_within(self.z8.codes(), z, ez)
        for buf, view, ld in ((self.zbuf, self.z, self.ldz), (self.gubuf, self.gu, self.ldgu)):
            b = buf.clone()
            b[self.skew: self.skew + self.M * ld].view(self.M, ld)[:, : view.shape[1]] = MARK
            assert bool((b == MARK).all())


SIZES = [(1, 1, 1), (1, 128, 128), (1, 130, 4096), (3, 77, 16), (16, 128, 32), (17, 129, 129), (32, 300, 640), (33, 256, 512), (64, 64, 1000), (65, 1000, 200),
         (128, 128, 384), (129, 515, 131), (256, 256, 256), (700, 333, 777), (1, 9000, 2048), (5, 40, 16384), (40, 2000, 4100), (100, 1100, 5000),
         (300, 5000, 1100), (2000, 4000, 300), (2500, 1300, 700), (20, 20000, 260)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("act,z_dtype", [("silu", F32), ("gelu", BF)], ids=["silu", "gelu"])
def test_forward(M, N, K, act, z_dtype):
    c = Forward(M, N, K, act, *inputs(M, N, K, M + N), z_dtype=z_dtype)
    c.run()
    c.check()


@pytest.mark.parametrize("M,N,K", [(3, 130, 700), (70, 260, 130), (300, 520, 1030)])
@pytest.mark.parametrize("z_dtype", [F32, BF])
@pytest.mark.parametrize("pad,skew", [(0, 4), (1, 1), (4, 0), (3, 2)])
def test_forward_strides_and_alignment(M, N, K, z_dtype, pad, skew):
    x, w = inputs(M, N, K, pad, ld=up(K, 16) + 16 * pad, lds=2 * N + M + pad)
    c = Forward(M, N, K, "silu", x, w, z_dtype, ldz=N + pad, ldgu=2 * N + pad, skew=skew, ldz8=up(N, 16) + 16 * pad, ldsz=M + pad)
    c.run()
    c.check()


def test_forward_with_fewer_results():
    c = Forward(100, 200, 300, "gelu", *inputs(100, 200, 300, 1))
    c.run()
    z, q, s, gu = c.z.clone(), c.z8.q.clone(), c.z8.s.clone(), c.gu.clone()
    for change in (dict(z=None), dict(gu=None), dict(z8=None, z_scale=None), dict(z=None, gu=None)):
        d = Forward(100, 200, 300, "gelu", c.x, c.w)
        d.run(**change)
        for name, x, y in (("z", z, d.z), ("gu", gu, d.gu), ("z8", q, d.z8.q), ("z8", s, d.z8.s)):
            assert torch.equal(x, y) == (name not in change)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M", [2, 200])
def test_forward_far_out_and_not_finite(act, M):
    """Gates of all sizes (up to thousands, where the activation is the gate or nothing), a whole block of zeros, and NaN."""
    N, K = 300, 256
    x, w = inputs(M, N, K, 7, scale=300.0)
    w.values[:128], w.q[:128] = 0.0, 0
    c = Forward(M, N, K, act, x, w)
    c.run()
    c.check()
    x.q[1, 5] = 0x7F                                  # one token is NaN, and the others are not
    w.q[N + 140, 9] = 0xFF                            # and one feature
    c.run()
    q, s = c.z8.codes()
    assert bool(torch.isnan(c.z[1]).all()) and (q[1] == 0x7F).all() and (s[1] == 0).all()
    rest = [m for m in range(M) if m != 1]
    assert bool(torch.isnan(c.z[rest, 140]).all()) and bool(torch.isfinite(c.z[rest][:, [n for n in range(N) if n != 140]]).all())
    assert (q[rest][:, 140] == 0x7F).all() and (q[rest, :128] & 127 == 0).all() and (q[rest][:, 141:] != 0x7F).all()


class Backward:
    def __init__(self, M, N, act, dz_dtype=BF, seed=0, ldgu=0, lddz=0, lddgu=0, skew=0, scale=1.5):
        g = torch.Generator().manual_seed(seed)
        self.M, self.N, self.kind, self.skew = M, N, act, skew
        self.ldgu, self.lddz, self.lddgu = ldgu or 2 * N, lddz or N, lddgu or 2 * N

        def matrix(x, ld, dtype):
            buf = torch.full((M * ld + skew + 32,), MARK, dtype=dtype, device="cuda")
            view = buf[skew: skew + M * ld].view(M, ld)[:, : x.shape[1]]
            view.copy_(x)
            return view

        self.gu, self.dz = matrix(torch.randn(M, 2 * N, generator=g) * scale, self.ldgu, BF), matrix(torch.randn(M, N, generator=g) * torch.randn(M, 1, generator=g).exp() * 1e-3, self.lddz, dz_dtype)
        self.dgu = matrix(torch.full((M, 2 * N), MARK), self.lddgu, BF)
        self.dq, self.dqt = Codes(M, 2 * N), Codes(2 * N, M)

    def args(self, **change):
        kw = dict(gu=self.gu, dz=self.dz, dz_dtype=KIND[self.dz.dtype], dq=self.dq.q, dq_scale=self.dq.s, dqt=self.dqt.q, dqt_scale=self.dqt.s, dgu=self.dgu,
                  ldgu=self.ldgu, lddz=self.lddz, lddgu=self.lddgu)
        return hp.make_gated_ffn_backward(self.M, self.N, ACT[self.kind], **{**kw, **change})

    def check(self):
        hp.hpsgd_gated_ffn_backward(self.args())
        torch.cuda.synchronize()
        gu, dz = self.gu.double().cpu().numpy(), self.dz.double().cpu().numpy()
        g, u = gu[:, : self.N], gu[:, self.N:]
        d = np.concatenate([dz * u * ref.slope(g, self.kind), dz * ref.act(g, self.kind)], axis=1)
        err = np.concatenate([np.abs(dz * u) * ref.slope_error(g, self.kind), np.abs(dz) * ref.act_error(g, self.kind)], axis=1) + np.abs(d) * 4 * E32 + 2.0 ** -126
        off = np.abs(self.dgu.double().cpu().numpy() - d) - err - E16 * (np.abs(d) + err)
        assert np.all(off <= 0), (off.max(), np.argwhere(off > 0)[:4])
        codes_within(self.dq.codes(), d, err)
        codes_within(self.dqt.codes(), np.ascontiguousarray(d.T), np.ascontiguousarray(err.T))
        b = self.dgu._base.clone()
        b[self.skew: self.skew + self.M * self.lddgu].view(self.M, self.lddgu)[:, : 2 * self.N] = MARK
        assert bool((b == MARK).all())


@pytest.mark.parametrize("M,N", [(1, 1), (3, 7), (1, 64), (128, 128), (130, 129), (127, 72), (200, 200), (513, 384), (300, 1000), (64, 2048), (1001, 136), (5, 4100)])
@pytest.mark.parametrize("act,dz_dtype", [("silu", BF), ("gelu", F32)], ids=["silu", "gelu"])
def test_backward(M, N, act, dz_dtype):
    Backward(M, N, act, dz_dtype, seed=M).check()


@pytest.mark.parametrize("N", [128, 200, 131])
@pytest.mark.parametrize("dz_dtype", [F32, BF])
@pytest.mark.parametrize("pad,skew", [(0, 1), (1, 0), (8, 8), (3, 2)])
def test_backward_strides_and_alignment(N, dz_dtype, pad, skew):
    Backward(150, N, "silu", dz_dtype, seed=pad, ldgu=2 * N + pad, lddz=N + pad, lddgu=2 * N + pad, skew=skew).check()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_backward_far_out_and_with_fewer_results(act):
    c = Backward(200, 256, act, scale=60.0)
    c.check()
    dq, dqt, dgu = c.dq.q.clone(), c.dqt.q.clone(), c.dgu.clone()
    for change in (dict(dq=None, dq_scale=None), dict(dqt=None, dqt_scale=None), dict(dgu=None), dict(dq=None, dq_scale=None, dqt=None, dqt_scale=None)):
        d = Backward(200, 256, act, scale=60.0)
        hp.hpsgd_gated_ffn_backward(d.args(**change))
        for name, x, y in (("dq", dq, d.dq.q), ("dqt", dqt, d.dqt.q), ("dgu", dgu, d.dgu)):
            assert torch.equal(x, y) == (name not in change)
    c.dz[3, 5] = float("inf")
    hp.hpsgd_gated_ffn_backward(c.args())
    q, _ = c.dq.codes()
    bad = np.zeros((200, 512), bool)
    bad[3, 5] = bad[3, 256 + 5] = True
    assert ((q & 127 == 127) <= bad).all() and (c.dqt.codes()[0] == 0x7F).sum() <= 2


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("N", [128, 100])
@pytest.mark.parametrize("dz_dtype", [F32, BF])
def test_backward_of_the_largest_gates(act, N, dz_dtype):
    """Where the sigmoid is 0 or 1 to binary32 the slope is too, whatever its other factors' sizes are: beside the bounds of the reference, 2^-112 (230 units, the most that
    g w' is where the sigmoid is 2^-126, and what the gate is held to there)."""
    sizes = np.array([0.0, 1.0, 9.0, 9.98, 10.06, 11.0, 50.0, 87.0, 88.5, 100.0, 1e4, 1e11, 1e15, 1.7e19, 1.9e19, 1e25, 1e30, 3e38])
    g = np.resize(np.concatenate([sizes, -sizes]), (5, N))
    gu = torch.ones(5, 2 * N, dtype=BF, device="cuda")
    gu[:, :N] = torch.from_numpy(g).to(BF)
    g = gu[:, :N].double().cpu().numpy()
    dgu = torch.full((5, 2 * N), MARK, dtype=BF, device="cuda")
    hp.hpsgd_gated_ffn_backward(hp.make_gated_ffn_backward(5, N, ACT[act], gu, torch.ones(5, N, dtype=dz_dtype, device="cuda"), KIND[dz_dtype], dgu=dgu))
    got = dgu.double().cpu().numpy()
    w, dw = ref.inner(g, act)
    s, r = ref.sigmoid(w), ref.sigmoid(-w)
    err = s * (r * (np.abs(w) * 2.0 ** -20.6 + 2.0 ** -22) + 2.0 ** -21) + np.abs(g * dw) * s * r * (np.abs(w) * 2.0 ** -19 + 2.0 ** -19.5) + 2.0 ** -112
    want = ref.slope(g, act)
    assert np.all(np.abs(got[:, :N] - want) <= err + E16 * (np.abs(want) + err))
    want, err = ref.act(g, act), np.abs(g) * s * (r * (np.abs(w) * 2.0 ** -20.6 + 2.0 ** -22) + 2.0 ** -21) + 2.0 ** -112
    assert np.all(np.abs(got[:, N:] - want) <= err + E16 * (np.abs(want) + err))


def test_the_same_bits_every_time_and_from_a_graph():
    M, N, K = 300, 640, 1100
    c, d = Forward(M, N, K, "silu", *inputs(M, N, K, 3)), Backward(M, N, "silu", seed=1)
    f, b = c.args(), d.args(gu=c.gu, ldgu=c.ldgu)

    def run():
        hp.hpsgd_gated_ffn_forward(f)
        hp.hpsgd_gated_ffn_backward(b)

    run()
    outs = (c.z, c.gu, *(x[:-64] for x in (c.z8.q, c.z8.s, d.dq.q, d.dq.s, d.dqt.q, d.dqt.s)), d.dgu)      # (64 marked bytes behind)
    first = [x.clone() for x in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for x in outs[:1] + outs[2:]:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    hp.hpsgd_ops_check()
    assert all(torch.equal(x, y) for x, y in zip(first, outs))
    c.x.q.copy_(c.x.q.flip(0))                         # other tokens in the same graph
    c.x.s.copy_(c.x.s.flip(1))
    d.dz.copy_(d.dz.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.z, first[0].flip(0)) and torch.equal(d.dgu, first[8].flip(0))


def test_offsets_beyond_2_to_the_31():
    M, N, K = 66_000, 17_000, 128                      # gu: 2.2 G elements
    rng = np.random.default_rng(0)
    x, w = Operand(rng.normal(size=(200, K))), Operand(rng.normal(size=(2 * N, K)) / 11.0)
    q, s = torch.zeros(M, K, dtype=U8, device="cuda"), torch.zeros(1, M, 4, dtype=U8, device="cuda")
    q[-200:], s[:, -200:] = x.q, x.s
    z8, zs, gu = torch.empty(M, up(N, 16), dtype=U8, device="cuda"), torch.empty(up(up(N, 128) // 128, 4) // 4, M, 4, dtype=U8, device="cuda"), torch.empty(M, 2 * N, dtype=BF, device="cuda")
    hp.hpsgd_gated_ffn_forward(hp.make_gated_ffn_forward(M, N, K, hp.HPSGD_SILU, q, s, w.q, w.s, z8=z8, z_scale=zs, gu=gu))
    c = Forward(200, N, K, "silu", x, w)
    c.run()
    assert torch.equal(gu[-200:], c.gu) and torch.equal(z8[-200:], c.z8.q[: 200 * c.z8.ld].view(200, -1)) and float(gu[: M - 200].abs().max()) == 0.0
    dz = torch.zeros(M, N, dtype=BF, device="cuda")
    dz[-200:] = torch.randn(200, N, device="cuda").to(BF)
    dq, ds = torch.empty(M, 2 * N, dtype=U8, device="cuda"), torch.empty(up(up(2 * N, 128) // 128, 4) // 4, M, 4, dtype=U8, device="cuda")
    hp.hpsgd_gated_ffn_backward(hp.make_gated_ffn_backward(M, N, hp.HPSGD_SILU, gu, dz, hp.HPSGD_BF16, dq=dq, dq_scale=ds))
    d1, s1 = torch.empty(200, 2 * N, dtype=U8, device="cuda"), torch.empty(up(up(2 * N, 128) // 128, 4) // 4, 200, 4, dtype=U8, device="cuda")
    hp.hpsgd_gated_ffn_backward(hp.make_gated_ffn_backward(200, N, hp.HPSGD_SILU, gu[-200:], dz[-200:], hp.HPSGD_BF16, dq=d1, dq_scale=s1))
    assert torch.equal(dq[-200:], d1) and torch.equal(ds[:, -200:], s1)
