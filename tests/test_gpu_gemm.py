"""hpsgd_gemm_fp8 against the product of the same codes and scales in binary64."""
import math

import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import ops_ref as ref

pytestmark = pytest.mark.gpu

U8, BF, F32 = torch.uint8, torch.bfloat16, torch.float32
KIND = {F32: hp.HPSGD_F32, BF: hp.HPSGD_BF16}
E32, E16 = 2.0 ** -24, 2.0 ** -8
TABLE = torch.from_numpy(ref.E4M3)


def up(n, a):
    return -(-n // a) * a


class Operand:
    """A random matrix in the block format: codes of every size, scales spread over many octaves.  What the format pads with, and what lies
    behind it, is filled with NaN codes and the largest scales: none of it may be read as data."""

    def __init__(self, rows, cols, seed, ld=0, lds=0, spread=8):
        g = torch.Generator().manual_seed(seed)
        self.ld, self.lds, nb = ld or up(cols, 16), lds or rows, up(cols, 128) // 128
        codes = torch.randint(0, 0x7F, (rows, cols), generator=g, dtype=torch.int64) | (torch.randint(0, 2, (rows, cols), generator=g) << 7)
        e = torch.randint(127 - spread, 128 + spread, (rows, nb), generator=g)
        q = torch.full((rows, self.ld), 0x7F, dtype=U8)
        q[:, :cols] = codes.to(U8)
        s = torch.full((up(nb, 4) // 4, self.lds, 4), 0xFE, dtype=U8)
        full = torch.full((rows, up(nb, 4)), 0xFE, dtype=torch.int64)
        full[:, :nb] = e
        s[:, :rows] = full.view(rows, -1, 4).permute(1, 0, 2).to(U8)
        self.q, self.s = q.cuda(), s.cuda()
        f = torch.ldexp(torch.ones(rows, nb, dtype=torch.float64), e - 127).repeat_interleave(128, dim=1)[:, :cols]
        self.values = (TABLE[codes] * f).cuda()


def product(M, N, K, a, b, d, **kw):
    ws = torch.full((hp.hpsgd_gemm_fp8_bytes(M, N, K),), 0xFF, dtype=U8, device="cuda")      # NaN, if it were read before it is written
    args = hp.make_gemm_fp8(M, N, K, a.q, a.s, b.q, b.s, d, KIND[d.dtype], workspace=ws, lda=a.ld, ldsa=a.lds, ldb=b.ld, ldsb=b.lds, **kw)
    hp.hpsgd_gemm_fp8(args)
    hp.hpsgd_ops_check()
    return args, ws


def check(d, a, b, K, before=None):
    """Binary32 sums of K exact products: each addition may be off by one unit in the last place of the sum of magnitudes (the tensor core may
    cut where it does not round, hence 2^-23), over at most K / 32 instructions and their 32 products, K / 4 being far above what either
    order needs."""
    want, mag = a.values @ b.values.t(), a.values.abs() @ b.values.abs().t()
    if before is not None:
        want, mag = want + before.double(), mag + before.double().abs()
    tol = 2 * E32 * (K / 4 + 8) * mag
    if d.dtype == BF:
        tol = tol + E16 * want.abs()
    err = (d.double() - want).abs()
    assert torch.all(err <= tol), float((err / tol.clamp(min=1e-300)).max())


SIZES = [(1, 1, 1), (1, 128, 128), (1, 130, 4096), (3, 77, 16), (16, 128, 32), (17, 129, 129), (32, 300, 640), (33, 256, 512), (64, 64, 1000),
         (65, 1000, 200), (128, 128, 384), (129, 515, 131), (200, 384, 1024), (256, 256, 256), (257, 1030, 2052), (700, 333, 777), (1, 30000, 256),
         (5, 40, 16384), (1000, 20000, 128)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("out", [F32, BF])
def test_product(M, N, K, out):
    a, b = Operand(M, K, 1), Operand(N, K, 2)
    d = torch.full((M, N), 3.0, dtype=out, device="cuda")
    product(M, N, K, a, b, d)
    check(d, a, b, K)


# Two, four and eight joined parts of even and uneven lengths on every width of tile; pairs of SMs, with a second tile for some of them and with
# fewer rows of B than one of them takes; sums in so many parts that they go through memory.
@pytest.mark.parametrize("M,N,K", [(1, 130, 2100), (2, 9000, 2048), (20, 4000, 2200), (40, 2000, 4100), (100, 1100, 5000), (300, 700, 3333), (1000, 1000, 2049),
                                   (1300, 2100, 1700), (2300, 4000, 1700), (18900, 130, 1700), (1, 100, 40000), (33, 200, 33000), (128, 128, 65536)])
@pytest.mark.parametrize("out", [F32, BF])
def test_product_in_parts_and_on_pairs(M, N, K, out):
    a, b = Operand(M, K, 21), Operand(N, K, 22)
    d = torch.full((M, N), math.nan, dtype=out, device="cuda")
    product(M, N, K, a, b, d)
    check(d, a, b, K)


@pytest.mark.parametrize("M,N,K", [(1, 130, 2100), (100, 1100, 5000), (1300, 2100, 1700), (3, 100, 40000)])
@pytest.mark.parametrize("skew", [0, 1, 4])
def test_parts_and_pairs_add_to_strided_results(M, N, K, skew):
    a, b = Operand(M, K, 23), Operand(N, K, 24)
    ldd = N + 2 + skew
    buf = torch.full((M * ldd + 16,), 7.0, device="cuda")
    d = buf[skew: skew + M * ldd].view(M, ldd)
    d[:, :N] = torch.randn(M, N, device="cuda") * 1e4
    before = d[:, :N].clone()
    product(M, N, K, a, b, d, ldd=ldd, accumulate=True)
    check(d[:, :N].contiguous(), a, b, K, before)
    product(M, N, K, a, b, d, ldd=ldd)
    check(d[:, :N].contiguous(), a, b, K)
    assert bool((d[:, N:] == 7).all()) and bool((buf[:skew] == 7).all()) and bool((buf[skew + M * ldd:] == 7).all())


@pytest.mark.parametrize("M,N,K", [(1, 130, 2100), (1000, 1000, 2049), (1300, 2100, 1700), (3, 100, 40000)])
def test_parts_and_pairs_repeat(M, N, K):
    a, b = Operand(M, K, 25), Operand(N, K, 26)
    d = torch.empty(M, N, device="cuda")
    args, ws = product(M, N, K, a, b, d)
    first = d.clone()
    for _ in range(20):
        d.fill_(math.nan)
        ws.fill_(0xFF)
        hp.hpsgd_gemm_fp8(args)
        assert torch.equal(d, first)


@pytest.mark.parametrize("M,N,K", [(1, 200, 2048), (100, 300, 4096), (300, 200, 260)])
def test_accumulate(M, N, K):
    a, b = Operand(M, K, 3), Operand(N, K, 4)
    d = torch.randn(M, N, device="cuda") * 1e4
    before = d.clone()
    product(M, N, K, a, b, d, accumulate=True)
    check(d, a, b, K, before)


@pytest.mark.parametrize("M,N,K", [(7, 100, 300), (150, 333, 1300)])
@pytest.mark.parametrize("out", [F32, BF])
@pytest.mark.parametrize("skew", [0, 1])
def test_strides(M, N, K, out, skew):
    a, b = Operand(M, K, 5, ld=up(K, 16) + 48, lds=M + 7), Operand(N, K, 6, ld=up(K, 16) + 16, lds=N + 1)
    buf = torch.full((M * (N + 5) + 16,), 7.0, device="cuda").to(out)
    d = buf[skew: skew + M * (N + 5)].view(M, N + 5)
    product(M, N, K, a, b, d, ldd=N + 5)
    check(d[:, :N].contiguous(), a, b, K)
    assert bool((d[:, N:] == 7).all()) and bool((buf[:skew] == 7).all()) and bool((buf[skew + M * (N + 5):] == 7).all())


def test_extreme_scales():
    """Scales from 2^-127 to 2^119: products from far below binary32's range to far above it."""
    M, N, K = 20, 140, 256
    a, b = Operand(M, K, 7, spread=0), Operand(N, K, 8, spread=0)          # values with scale 1
    a.s[:] = 0
    b.s[:] = 0
    d = torch.full((M, N), 3.0, device="cuda")
    product(M, N, K, a, b, d)
    assert bool((d == 0).all())
    a.s[:] = 246
    d2 = torch.empty_like(d)
    product(M, N, K, a, b, d2)                                   # 2^119 * 2^-127 = 2^-8
    want, mag = (x * 2.0 ** -8 for x in (a.values @ b.values.t(), a.values.abs() @ b.values.abs().t()))
    assert torch.all((d2.double() - want).abs() <= 2 * E32 * 72 * mag)
    b.s[:] = 246
    product(M, N, K, a, b, d2)
    big = (a.values @ b.values.t()).abs() > 1
    assert bool(torch.isinf(d2[big]).all())


def test_nan_codes_reach_their_row_and_column_only():
    M, N, K = 40, 200, 500
    a, b = Operand(M, K, 9), Operand(N, K, 10)
    a.q[11, 499] = 0x7F
    b.q[150, 3] = 0xFF
    d = torch.empty(M, N, device="cuda")
    product(M, N, K, a, b, d)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[11], bad[:, 150] = True, True
    assert bool(torch.isnan(d[bad]).all()) and bool(torch.isfinite(d[~bad]).all())


@pytest.mark.parametrize("M,N,K", [(1, 256, 8192), (100, 100, 8192), (256, 256, 1024)])
def test_workspace_serves_call_after_call_and_results_repeat(M, N, K):
    a, b, c = Operand(M, K, 11), Operand(N, K, 12), Operand(M, K, 13)
    d = torch.empty(M, N, device="cuda")
    args, ws = product(M, N, K, a, b, d)
    first = d.clone()
    e = torch.empty(M, N, device="cuda")
    other = hp.make_gemm_fp8(M, N, K, c.q, c.s, b.q, b.s, e, 0, workspace=ws)
    for _ in range(20):
        d.fill_(math.nan)
        hp.hpsgd_gemm_fp8(other)
        hp.hpsgd_gemm_fp8(args)
        assert torch.equal(d, first)
    check(e, c, b, K)


def test_nothing_to_do():
    d = torch.full((4, 8), 5.0, device="cuda")
    hp.hpsgd_gemm_fp8(hp.make_gemm_fp8(4, 6, 0, None, None, None, None, d, 0, ldd=8))
    assert bool((d[:, :6] == 0).all()) and bool((d[:, 6:] == 5).all())
    hp.hpsgd_gemm_fp8(hp.make_gemm_fp8(4, 6, 0, None, None, None, None, d, 0, ldd=8, accumulate=True))
    assert bool((d[:, :6] == 0).all())


def test_captured_and_on_a_stream_of_its_own():
    M, N, K = 1, 512, 4096
    a, b = Operand(M, K, 14), Operand(N, K, 15)
    d = torch.zeros(M, N, device="cuda")
    args, ws = product(M, N, K, a, b, d)
    want = d.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hp.hpsgd_gemm_fp8(args, stream=torch.cuda.current_stream())
    d.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(d, want)


def test_a_linear_layer_s_three_products():
    """Forward, input gradient and weight gradient through the quantiser, against the binary64 products of what the codes stand for; and the
    whole against the unquantised products: each code is off by at most 2^-4 of its value, so are the products by 2 * 2^-4 and a little of
    their magnitudes' sum."""
    M, N, K = 200, 300, 400
    torch.manual_seed(0)
    x, w, dy = torch.randn(M, K, device="cuda"), 0.05 * torch.randn(N, K, device="cuda"), 1e-3 * torch.randn(M, N, device="cuda")

    def quantize(v, transposed=True):
        r, c = v.shape
        q = torch.zeros(r, up(c, 16), dtype=U8, device="cuda")
        s = torch.zeros(up(up(c, 128) // 128, 4) // 4, r, 4, dtype=U8, device="cuda")
        qt = torch.zeros(c, up(r, 16), dtype=U8, device="cuda")
        st = torch.zeros(up(up(r, 128) // 128, 4) // 4, c, 4, dtype=U8, device="cuda")
        hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(r, c, 0, v, q=q, scale=s, qt=qt, scale_t=st))
        return (q, s), (qt, st)

    (xq, xt), (wq, wt), (gq, gt) = quantize(x), quantize(w), quantize(dy)
    for m, n, k, a, b, want, mag in ((M, N, K, xq, wq, x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()),
                                     (M, K, N, gq, wt, dy.double() @ w.double(), dy.double().abs() @ w.double().abs()),
                                     (N, K, M, gt, xt, dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs())):
        d = torch.empty(m, n, device="cuda")
        ws = torch.zeros(hp.hpsgd_gemm_fp8_bytes(m, n, k), dtype=U8, device="cuda")
        hp.hpsgd_gemm_fp8(hp.make_gemm_fp8(m, n, k, *a, *b, d, 0, workspace=ws))
        assert torch.all((d.double() - want).abs() <= 0.13 * mag)
        # random signs: the errors' root mean square is far smaller
        assert float((d.double() - want).norm() / want.norm()) < 0.06
