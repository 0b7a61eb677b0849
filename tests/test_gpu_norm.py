"""hpsgd_rmsnorm_forward / _backward and hpsgd_quantize_fp8 against their definitions in binary64."""
import math

import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import ops_ref as ref

pytestmark = pytest.mark.gpu

U8, BF, F32 = torch.uint8, torch.bfloat16, torch.float32
KIND = {F32: hp.HPSGD_F32, BF: hp.HPSGD_BF16}
E32, E16 = 2.0 ** -24, 2.0 ** -8        # unit roundoffs of 24 and 8 significant bits


def up(n, a):
    return -(-n // a) * a


class Codes:
    """Room for a matrix in the block format with everything around it marked."""

    def __init__(self, rows, cols, ld=0, lds=0):
        self.rows, self.cols, self.ld, self.lds = rows, cols, ld or up(cols, 16), lds or rows
        self.words = up(up(cols, 128) // 128, 4) // 4
        self.q = torch.full((rows * self.ld + 64,), 0xA5, dtype=U8, device="cuda")
        self.s = torch.full((self.words * self.lds * 4 + 64,), 0xA5, dtype=U8, device="cuda")

    def codes(self):
        """Codes and scale bytes; checks the zeros behind the last column and block, and that nothing else was touched."""
        q = self.q.cpu().numpy()
        assert (q[self.rows * self.ld:] == 0xA5).all()
        q = q[: self.rows * self.ld].reshape(self.rows, self.ld)
        pad = up(self.cols, 16)
        assert (q[:, self.cols: pad] == 0).all() and (q[:, pad:] == 0xA5).all()
        s = self.s.cpu().numpy()
        n = self.words * self.lds * 4
        assert (s[n:] == 0xA5).all()
        s = s[:n].reshape(self.words, self.lds, 4)
        assert (s[:, self.rows:] == 0xA5).all()
        s = s[:, : self.rows].transpose(1, 0, 2).reshape(self.rows, -1)
        nb = up(self.cols, 128) // 128
        assert (s[:, nb:] == 0).all()
        return q[:, : self.cols], s[:, :nb].astype(np.int64)


def same_codes(got, x, rel):
    """Codes and scales of x, where x is known to within `rel` of itself: the same scale unless the block's top is that near to the edge of
    two scales, and then the nearest code unless x is that near to the middle of two."""
    q, e = got
    want_e = ref.scale_bytes(np.abs(ref.blocks(np.where(np.isfinite(x), x, 0.0))).max(axis=2))
    top = np.abs(ref.blocks(np.where(np.isfinite(x), x, 0.0))).max(axis=2)
    edge = np.abs(top / (448 * ref.factor(np.minimum(want_e, e))) - 1) <= 2 * rel
    assert np.all((e == want_e) | edge)
    f = np.repeat(ref.factor(e), 128, axis=1)[:, : x.shape[1]]
    v = ref.E4M3[q]
    bad = ~np.isfinite(x)
    assert np.all(q[bad] == 0x7F)
    x, v, f = x[~bad], v[~bad], f[~bad]
    y = np.clip(x / f, -448, 448)
    want = ref.E4M3[ref.nearest_code(y)]
    off = v != want
    assert np.all(np.abs(np.abs(y - v) - np.abs(y - want))[off] <= 4 * rel * np.abs(y[off]) + 1e-12)


def strided(rows, cols, ld, dtype, skew=0, fill=7.0):
    buf = torch.full((rows * ld + skew + 64,), fill, device="cuda").to(dtype)
    return buf, buf[skew: skew + rows * ld].view(rows, ld)[:, :cols]


def outside_untouched(buf, view, skew, rows, ld, fill=7.0):
    b = buf.clone()
    b[skew: skew + rows * ld].view(rows, ld)[:, : view.shape[1]] = fill
    assert bool((b == fill).all())


SHAPES = [(1, 1), (1, 1024), (3, 7), (2, 8), (5, 127), (4, 128), (3, 129), (7, 511), (2, 512), (3, 513), (2, 1000), (130, 1032), (3, 2056),
          (2, 4096), (2, 4104), (2, 8200), (1, 16384), (700, 72)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,wdtype", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("residual", [True, False])
def test_forward(rows, cols, dtype, wdtype, residual):
    torch.manual_seed(rows * 7 + cols)
    x = (torch.randn(rows, cols, device="cuda") * torch.randn(cols, device="cuda").exp()).to(dtype)
    res = torch.randn(rows, cols, device="cuda").to(dtype) if residual else None
    w = (1 + 0.2 * torch.randn(cols, device="cuda")).to(wdtype)
    h = torch.empty_like(x) if residual else None
    y, rstd, c = torch.empty_like(x), torch.empty(rows, device="cuda"), Codes(rows, cols)
    a = hp.make_rmsnorm_forward(rows, cols, 1e-5, KIND[dtype], x, w, residual=res, h=h, y=y, y8=c.q, y_scale=c.s, rstd=rstd, weight_dtype=KIND[wdtype])
    hp.hpsgd_rmsnorm_forward(a)
    h64 = x.double()
    if residual:
        s = x.double() + res.double()
        assert torch.all((h.double() - s).abs() <= s.abs() * (E16 if dtype == BF else E32) + 1e-40)
        h64 = h.double()
    want_r = 1 / torch.sqrt((h64 * h64).mean(dim=1) + 1e-5)
    # a sum of n squares in a tree of at most 32 sequential terms a thread and 12 levels, halved by the root; division and root
    assert torch.all((rstd.double() - want_r).abs() <= 26 * E32 * want_r)
    want = h64 * want_r[:, None] * w.double()
    assert torch.all((y.double() - want).abs() <= want.abs() * ((E16 if dtype == BF else 0) + 30 * E32))
    same_codes(c.codes(), want.cpu().numpy(), 30 * E32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cols,ld,skew", [(130, 137, 0), (130, 136, 1), (256, 264, 0), (1001, 1016, 8), (64, 64, 3)])
def test_forward_strides_and_alignment(dtype, cols, ld, skew):
    rows = 9
    torch.manual_seed(cols)
    bx, x = strided(rows, cols, ld, dtype, skew)
    br, r = strided(rows, cols, ld + 8, dtype, skew)
    bh, h = strided(rows, cols, ld + 3, dtype, skew)
    by, y = strided(rows, cols, ld, dtype, skew)
    x.copy_(torch.randn(rows, cols, device="cuda"))
    r.copy_(torch.randn(rows, cols, device="cuda"))
    w = torch.randn(cols + 1, device="cuda").to(dtype)[1:]
    c = Codes(rows, cols, ld=up(cols, 16) + 32, lds=rows + 5)
    a = hp.make_rmsnorm_forward(rows, cols, 0.0, KIND[dtype], x, w, residual=r, h=h, y=y, y8=c.q, y_scale=c.s, ldx=ld, ldres=ld + 8, ldh=ld + 3, ldy=ld,
                                ldy8=c.ld, ldys=c.lds)
    hp.hpsgd_rmsnorm_forward(a)
    h64 = h.double()
    want = h64 / torch.sqrt((h64 * h64).mean(dim=1, keepdim=True)) * w.double()
    assert torch.equal(h, (x.float() + r.float()).to(dtype))
    assert torch.all((y.double() - want).abs() <= want.abs() * ((E16 if dtype == BF else 0) + 30 * E32))
    same_codes(c.codes(), want.cpu().numpy(), 30 * E32)
    outside_untouched(bh, h, skew, rows, ld + 3)
    outside_untouched(by, y, skew, rows, ld)


def test_forward_in_place_and_one_output_only():
    x, r, w = (torch.randn(50, 300, device="cuda").to(BF) for _ in range(3))
    w = w[0].contiguous()
    want = (x.float() + r.float()).to(BF)
    for target in ("x", "residual"):
        x2, r2 = x.clone(), r.clone()
        y = torch.empty_like(x)
        h = x2 if target == "x" else r2
        hp.hpsgd_rmsnorm_forward(hp.make_rmsnorm_forward(50, 300, 1e-5, hp.HPSGD_BF16, x2, w, residual=r2, h=h, y=y))
        assert torch.equal(h, want)


def test_forward_rows_of_zeros_and_rows_that_are_not_finite():
    x = torch.randn(6, 200, device="cuda")
    x[1] = 0.0
    x[2, 5] = math.inf
    x[3, 199] = math.nan
    x[4, 130] = -3e38
    w = torch.ones(200, device="cuda")
    c, rstd, y = Codes(6, 200), torch.empty(6, device="cuda"), torch.empty_like(x)
    hp.hpsgd_rmsnorm_forward(hp.make_rmsnorm_forward(6, 200, 1e-5, hp.HPSGD_F32, x, w, y8=c.q, y_scale=c.s, rstd=rstd, y=y))
    q, e = c.codes()
    assert (q[1] == 0).all() and (e[1] == 0).all() and abs(rstd[1].item() - 1e5 ** 0.5) < 1e-3
    # inf: rstd is 0, everything becomes 0 but the infinity itself (inf * 0); NaN: everything; 3e38: its square is inf in binary32
    assert q[2, 5] == 0x7F and (np.delete(q[2], 5) & 0x7F == 0).all()
    assert (q[3] == 0x7F).all() and (q[4] & 0x7F == 0).all()
    assert np.isfinite(ref.E4M3[q[[0, 5]]]).all()


@pytest.mark.parametrize("rows,cols", SHAPES + [(592, 40), (593, 40), (3000, 264)])
@pytest.mark.parametrize("dtype,wdtype", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("residual", [True, False])
def test_backward(rows, cols, dtype, wdtype, residual):
    torch.manual_seed(rows * 7 + cols)
    h = (torch.randn(rows, cols, device="cuda") * torch.randn(cols, device="cuda").exp()).to(dtype)
    dy = torch.randn(rows, cols, device="cuda").to(dtype)
    dres = torch.randn(rows, cols, device="cuda").to(dtype) if residual else None
    w = (1 + 0.2 * torch.randn(cols, device="cuda")).to(wdtype)
    rstd = torch.rsqrt(h.float().square().mean(dim=1) + 1e-5)
    dx, dw = torch.empty_like(h), torch.full((cols,), 9.0, device="cuda")
    ws = torch.full((hp.hpsgd_rmsnorm_backward_bytes(rows, cols),), 0xFF, dtype=U8, device="cuda")      # NaN, if it were read
    a = hp.make_rmsnorm_backward(rows, cols, KIND[dtype], h, w, rstd, dy, dx, dw, ws, dres=dres, weight_dtype=KIND[wdtype])
    hp.hpsgd_rmsnorm_backward(a)
    r = rstd.double()[:, None]
    xn, d = h.double() * r, dy.double() * w.double()
    mean = (d * xn).mean(dim=1, keepdim=True)
    want = r * (d - xn * mean)
    scale = r * (d.abs() + xn.abs() * (d * xn).abs().mean(dim=1, keepdim=True))     # the terms' magnitudes bound the cancellation
    if residual:
        want, scale = want + dres.double(), scale + dres.double().abs()
    assert torch.all((dx.double() - want).abs() <= 40 * E32 * scale + (E16 * want.abs() if dtype == BF else 0))
    want_w, mag = (dy.double() * xn).sum(dim=0), (dy.double() * xn).abs().sum(dim=0)
    # rows of a block one after the other, then up to 74 partial sums, then 8
    assert torch.all((dw.double() - want_w).abs() <= (min(rows, rows / 592 + 1) + 90) * E32 * mag)


def test_backward_agrees_with_differences():
    """Directional derivative of sum(y * g) through the forward call's own fp32 output."""
    rows, cols = 5, 96
    torch.manual_seed(3)
    x, u, g = (torch.randn(rows, cols, device="cuda") for _ in range(3))
    w, v = 1 + 0.1 * torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")

    def loss(x, w):
        y, r = torch.empty_like(x), torch.empty(rows, device="cuda")
        hp.hpsgd_rmsnorm_forward(hp.make_rmsnorm_forward(rows, cols, 1e-5, 0, x.contiguous(), w.contiguous(), y=y, rstd=r))
        return (y.double() * g.double()).sum().item(), r

    _, r = loss(x, w)
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    ws = torch.empty(hp.hpsgd_rmsnorm_backward_bytes(rows, cols), dtype=U8, device="cuda")
    hp.hpsgd_rmsnorm_backward(hp.make_rmsnorm_backward(rows, cols, 0, x, w, r, g, dx, dw, ws))
    t = 1e-2
    # central difference: t^2 of third derivatives (magnitudes of order 10) and binary32 noise of 500 outputs over 2 t
    num = (loss(x + t * u, w)[0] - loss(x - t * u, w)[0]) / (2 * t)
    assert abs(num - (dx.double() * u.double()).sum().item()) < 0.02
    num = (loss(x, w + t * v)[0] - loss(x, w - t * v)[0]) / (2 * t)
    assert abs(num - (dw.double() * v.double()).sum().item()) < 0.01


@pytest.mark.parametrize("target", ["dy", "dres"])
@pytest.mark.parametrize("cols", [200, 3000, 9000])
def test_backward_in_place_and_strided(target, cols):
    rows, ld = 20, cols + 5
    _, h = strided(rows, cols, ld, BF)
    _, dy = strided(rows, cols, ld + 1, BF)
    _, dr = strided(rows, cols, ld + 2, BF)
    for x in (h, dy, dr):
        x.copy_(torch.randn(rows, cols, device="cuda"))
    w = torch.randn(cols, device="cuda").to(BF)
    rstd = torch.rsqrt(h.float().square().mean(dim=1))
    out = []
    for place in (False, True):
        dy2, dr2 = dy.contiguous(), dr.contiguous()
        dx = torch.empty(rows, cols, dtype=BF, device="cuda") if not place else dy2 if target == "dy" else dr2
        dw = torch.empty(cols, device="cuda")
        ws = torch.empty(hp.hpsgd_rmsnorm_backward_bytes(rows, cols), dtype=U8, device="cuda")
        hp.hpsgd_rmsnorm_backward(hp.make_rmsnorm_backward(rows, cols, hp.HPSGD_BF16, h, w, rstd, dy2, dx, dw, ws, dres=dr2, ldh=ld))
        out.append((dx.clone(), dw))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    dx, dw = torch.empty(rows, cols, dtype=BF, device="cuda"), torch.empty(cols, device="cuda")
    hp.hpsgd_rmsnorm_backward(hp.make_rmsnorm_backward(rows, cols, hp.HPSGD_BF16, h, w, rstd, dy, dx, dw, ws, dres=dr, ldh=ld, lddy=ld + 1, lddres=ld + 2))
    assert torch.equal(out[0][0], dx) and torch.equal(out[0][1], dw)


def test_backward_without_rows():
    dw = torch.full((40,), 3.0, device="cuda")
    hp.hpsgd_rmsnorm_backward(hp.make_rmsnorm_backward(0, 40, 0, None, None, None, None, None, dw, None))
    assert bool((dw == 0).all())


# ---------------------------------------------------------------------------------------------- quantisation
QSHAPES = [(1, 1), (1, 300), (300, 1), (16, 16), (127, 129), (128, 128), (129, 127), (130, 515), (385, 64), (512, 640)]


def spread(rows, cols):
    torch.manual_seed(rows + 31 * cols)
    return torch.randn(rows, cols, device="cuda") * torch.randn(rows, 1, device="cuda").mul(4).exp() * torch.randn(cols, device="cuda").exp()


@pytest.mark.parametrize("rows,cols", QSHAPES)
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("which", ["both", "rows", "columns"])
def test_quantize(rows, cols, dtype, which):
    x = spread(rows, cols).to(dtype)
    a, b = Codes(rows, cols), Codes(cols, rows)
    kw = {}
    if which != "columns":
        kw |= dict(q=a.q, scale=a.s)
    if which != "rows":
        kw |= dict(qt=b.q, scale_t=b.s)
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(rows, cols, KIND[dtype], x, **kw))
    x = x.double().cpu().numpy()
    for c, v in ([(a, x)] if which != "columns" else []) + ([(b, x.T)] if which != "rows" else []):
        q, e = c.codes()
        want_q, want_e = ref.quantize(v)
        assert np.array_equal(e, want_e) and np.array_equal(q & 0x7F, want_q & 0x7F)       # powers of two: nothing is rounded before the code
        assert np.array_equal(ref.E4M3[q], ref.E4M3[want_q])


@pytest.mark.parametrize("rows,cols", QSHAPES)
def test_transpose_of_a_matrix_in_the_format(rows, cols):
    x = spread(rows, cols)
    a, b = Codes(rows, cols, lds=rows + 3), Codes(cols, rows, ld=up(rows, 16) + 16, lds=cols + 1)
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(rows, cols, 0, x, q=a.q, scale=a.s, lds=a.lds))
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(rows, cols, hp.HPSGD_FP8, a.q, x_scale=a.s, ldxs=a.lds, qt=b.q, scale_t=b.s, ldqt=b.ld, ldst=b.lds))
    v = ref.values(*a.codes())
    q, e = b.codes()
    want_q, want_e = ref.quantize(v.T)
    assert np.array_equal(e, want_e) and np.array_equal(ref.E4M3[q], ref.E4M3[want_q])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("ld,skew", [(141, 0), (144, 1), (136, 8)])
def test_quantize_strides_and_alignment(dtype, ld, skew):
    rows, cols = 140, 133
    _, x = strided(rows, cols, ld, dtype, skew)
    x.copy_(spread(rows, cols))
    a, b = Codes(rows, cols, ld=160, lds=200), Codes(cols, rows, ld=176, lds=150)
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(rows, cols, KIND[dtype], x, ldx=ld, q=a.q, scale=a.s, ldq=160, lds=200, qt=b.q, scale_t=b.s, ldqt=176, ldst=150))
    v = x.double().cpu().numpy()
    for c, u in ((a, v), (b, v.T)):
        q, e = c.codes()
        want_q, want_e = ref.quantize(u)
        assert np.array_equal(e, want_e) and np.array_equal(ref.E4M3[q], ref.E4M3[want_q])


def test_quantize_values_at_the_edges():
    """Zeros, the largest and smallest binary32 numbers, exact scale edges, ties, infinities and NaN."""
    x = np.zeros((8, 256), dtype=np.float32)
    x[1, 0], x[1, 130] = 3.4028235e38, -1e-45
    x[2, :128] = np.float32(2.0 ** -149) * np.arange(128)
    x[3, 0], x[3, 128] = 448.0, np.nextafter(np.float32(448.0), np.float32(1000.0))
    x[4, :128] = np.linspace(0, 31.75, 128)                     # every quarter: ties of the coarser codes
    x[4, 127] = 448.0
    x[5, 3], x[5, 4], x[5, 5], x[5, 6] = math.inf, -math.inf, math.nan, 2.0
    x[6, 128:] = math.nan
    x[7, 0], x[7, 1] = -448.0 * 2.0 ** -127, 2.0 ** -136
    a, b = Codes(8, 256), Codes(256, 8)
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(8, 256, 0, torch.from_numpy(x).cuda(), q=a.q, scale=a.s, qt=b.q, scale_t=b.s))
    for c, v in ((a, x.astype(np.float64)), (b, x.T.astype(np.float64))):
        q, e = c.codes()
        want_q, want_e = ref.quantize(v)
        assert np.array_equal(e, want_e)
        assert np.array_equal(np.isnan(ref.E4M3[q]), np.isnan(ref.E4M3[want_q]))
        assert np.array_equal(np.nan_to_num(ref.E4M3[q]), np.nan_to_num(ref.E4M3[want_q]))
