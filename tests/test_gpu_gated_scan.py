"""hpsgd_gated_scan_forward / _backward against the recurrence in binary64."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp
from tests import scan_ref as ref

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
KIND = {F32: hp.HPSGD_F32, BF: hp.HPSGD_BF16}
HALF = {F32: 2.0 ** -24, BF: 2.0 ** -8}            # half a step, relative to the value
MARK = 77.0


def up(n, a):
    return -(-n // a) * a


class Case:
    """Inputs, marked outputs and the calls of one shape.  `bounds`: rows at which sequences begin, and the end; None: equal sequences.
    `side`: f, v and o in one matrix; `pad`: more columns in every row."""

    def __init__(self, rows, cols, sequences, bounds=None, dtype=F32, gate=True, states=True, pad=0, shift=0, seed=0, bias=3.0):
        self.rows, self.cols, self.n, self.dtype, self.gate, self.states = rows, cols, sequences, dtype, gate, states
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.ld = cols + pad
        self.bounds = list(bounds) if bounds is not None else [k * (rows // max(1, sequences)) for k in range(sequences + 1)]
        self.offsets = torch.tensor(bounds, dtype=torch.int64, device="cuda") if bounds is not None else None

        def matrix(x):
            """On the device, `shift` elements behind a wide boundary, rows self.ld apart."""
            flat = torch.full((shift + max(1, rows) * self.ld + 8,), MARK, dtype=dtype, device="cuda")
            view = flat[shift: shift + rows * self.ld].view(rows, self.ld)[:, :cols]
            view.copy_(x.to(dtype))
            return view

        self.f, self.v, self.dy = matrix(rnd(rows, cols) * 1.5 + bias * torch.rand(cols, generator=g)), matrix(rnd(rows, cols)), matrix(rnd(rows, cols))
        self.o = matrix(rnd(rows, cols) * 2.0) if gate else None
        self.h0 = rnd(sequences, cols).cuda() if states else None
        self.dh_last = rnd(sequences, cols).cuda() if states else None
        mark = torch.full((rows, cols), MARK)
        self.y, self.df, self.dv, self.do = matrix(mark), matrix(mark), matrix(mark), matrix(mark) if gate else None
        self.h_last = torch.full((sequences, cols), MARK, device="cuda") if states else None
        self.dh0 = torch.full((sequences, cols), MARK, device="cuda") if states else None
        self.saved = torch.full((hp.hpsgd_gated_scan_saved_bytes(rows, cols) // 4 + 8,), float("nan"), device="cuda")

    def forward(self, **change):
        kw = dict(f=self.f, v=self.v, o=self.o, y=self.y, offsets=self.offsets, h0=self.h0, h_last=self.h_last, saved=self.saved,
                  ldf=self.ld, ldv=self.ld, ldo=self.ld, ldy=self.ld)
        return hp.make_gated_scan_forward(self.rows, self.cols, self.n, KIND[self.dtype], **{**kw, **change})

    def backward(self, **change):
        kw = dict(f=self.f, v=self.v, o=self.o, saved=self.saved, dy=self.dy, df=self.df, dv=self.dv, do=self.do, offsets=self.offsets, h0=self.h0,
                  dh_last=self.dh_last, dh0=self.dh0, ldf=self.ld, ldv=self.ld, ldo=self.ld, lddy=self.ld, lddf=self.ld, lddv=self.ld, lddo=self.ld)
        return hp.make_gated_scan_backward(self.rows, self.cols, self.n, KIND[self.dtype], **{**kw, **change})

    def host(self):
        d = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        return d(self.f), d(self.v), d(self.o), self.bounds, d(self.h0)

    def check(self):
        hp.hpsgd_gated_scan_forward(self.forward())
        hp.hpsgd_gated_scan_backward(self.backward())
        torch.cuda.synchronize()
        inside = np.zeros(self.rows, dtype=bool)
        inside[self.bounds[0]: self.bounds[-1]] = True
        d = lambda x: x.double().cpu().numpy()  # noqa: E731
        want = ref.forward(*self.host())
        back = ref.backward(*self.host(), d(self.dy), None if self.dh_last is None else d(self.dh_last))

        def rows_of(name, got, value, err):
            got = d(got)
            assert (got[~inside] == MARK).all(), name
            x, e = value[inside], err[inside]
            # (a gate is not held below 2^-126; no product it enters here is above 64)
            off = np.abs(got[inside] - x) - e - HALF[self.dtype] * (np.abs(x) + e) - 2.0 ** -120
            assert (off <= 0).all(), (name, off.max(), np.argwhere(off > 0)[:4])

        rows_of("y", self.y, want["y"], want["y_err"])
        rows_of("df", self.df, back["df"], back["df_err"])
        rows_of("dv", self.dv, back["dv"], back["dv_err"])
        if self.gate:
            rows_of("do", self.do, back["do"], back["do_err"])
        if self.states:
            assert (np.abs(d(self.h_last) - want["h_last"]) <= want["h_last_err"]).all()
            assert (np.abs(d(self.dh0) - back["dh0"]) <= back["dh0_err"]).all()
        for x in (self.f, self.y, self.df):         # nothing beside the columns and behind the rows
            whole = x._base if x._base is not None else x
            if self.ld > self.cols:
                assert float((x.as_strided((self.rows, self.ld - self.cols), (self.ld, 1), x.storage_offset() + self.cols).float() - MARK).abs().max()) == 0.0
            assert float((whole.view(-1)[-8:].float() - MARK).abs().max()) == 0.0


SHAPES = [(1, 1, 1), (1, 2, 1), (3, 64, 3), (2, 130, 1), (7, 3, 1), (16, 64, 1), (17, 65, 1), (128, 66, 2), (129, 64, 1), (300, 31, 5), (1025, 128, 1),
          (2048, 64, 2), (4100, 72, 4), (640, 200, 640), (96, 9600, 2), (300, 9602, 1)]


@pytest.mark.parametrize("rows,cols,sequences", SHAPES)
@pytest.mark.parametrize("dtype,gate,states", [(F32, True, True), (BF, False, False), (BF, True, True)], ids=["f32", "bf16 plain", "bf16"])
def test_equal_sequences(rows, cols, sequences, dtype, gate, states):
    Case(rows, cols, sequences, dtype=dtype, gate=gate, states=states, seed=rows + cols).check()


RAGGED = {"behind and in front": (1000, [13, 200, 201, 640, 900]), "empty ones": (500, [0, 0, 0, 100, 100, 100, 101, 400, 400, 400]),
          "all empty": (40, [7, 7, 7]), "one row each": (600, list(range(601))), "nothing": (64, [0, 0]), "aligned": (1024, [0, 128, 256, 512, 1024]),
          "next to the edges": (1024, [0, 15, 16, 17, 127, 128, 129, 1023, 1024]), "one long": (3000, [0, 1, 2, 3, 2999, 3000])}


@pytest.mark.parametrize("name", RAGGED)
@pytest.mark.parametrize("cols", [64, 37, 2500])
@pytest.mark.parametrize("dtype,gate,states", [(F32, False, True), (BF, True, True)], ids=["f32", "bf16"])
def test_ragged_sequences(name, cols, dtype, gate, states):
    rows, bounds = RAGGED[name]
    Case(rows, cols, len(bounds) - 1, bounds=bounds, dtype=dtype, gate=gate, states=states, seed=len(name)).check()


def test_many_ragged_sequences():
    """More sequences than a warp looks at in one step of its search, among them runs of empty ones longer than that."""
    rng = np.random.default_rng(5)
    for empty, cuts in ((0, 32), (70, 1029)):
        bounds = sorted([0, 1990] + rng.integers(0, 1990, cuts).tolist() + [777] * empty)
        Case(2000, 64, len(bounds) - 1, bounds=bounds, seed=cuts).check()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("pad,shift", [(1, 0), (2, 0), (0, 1), (6, 2), (3, 1)])
def test_strides_and_alignment(dtype, pad, shift):
    Case(150, 66, 3, dtype=dtype, pad=pad, shift=shift, seed=pad).check()
    Case(150, 67, 3, dtype=dtype, pad=pad, shift=shift, seed=pad).check()


def test_gates_that_are_open_or_shut():
    """Gates far out: nothing forgotten for 3000 rows, nothing kept, and both in turn."""
    c = Case(3000, 64, 1, dtype=F32, seed=9)
    c.f[:, :16] = 40.0
    c.f[:, 16:32] = -40.0
    c.f[::2, 32:48] = 120.0
    c.f[1::2, 32:48] = -120.0
    c.check()
    assert torch.equal(c.y[:, 16:32], (c.v * torch.sigmoid(c.o))[:, 16:32]) or float((c.y[:, 16:32] - (c.v * torch.sigmoid(c.o))[:, 16:32]).abs().max()) < 1e-5
    c.f[:, :32] = float("inf")
    c.f[:, 32:] = float("-inf")
    hp.hpsgd_gated_scan_forward(c.forward())
    hp.hpsgd_gated_scan_backward(c.backward())
    torch.cuda.synchronize()
    assert torch.equal(c.h_last[0, :32], c.h0[0, :32]) and torch.equal(c.h_last[0, 32:], c.v[-1, 32:])
    for x in (c.y, c.df, c.dv, c.do, c.dh0):
        assert bool(torch.isfinite(x).all())
    assert float(c.dv[:, :32].abs().max()) == 0.0


@pytest.mark.parametrize("cols", [64, 2500])
def test_what_is_not_finite_stays_in_its_sequence(cols):
    bounds = [0, 300, 301, 500, 900, 1200]
    c, clean = (Case(1200, cols, 5, bounds=bounds, seed=3) for _ in range(2))
    c.v[100, 3], c.f[310, 1], c.h0[3, 2], c.dy[1000, 0] = float("nan"), float("nan"), float("inf"), float("nan")
    for k in (c, clean):
        hp.hpsgd_gated_scan_forward(k.forward())
        hp.hpsgd_gated_scan_backward(k.backward())
    torch.cuda.synchronize()
    for rows, col in ((slice(0, 300), 3), (slice(301, 500), 1), (slice(500, 900), 2), (slice(900, 1200), 0)):
        for name in ("y", "df", "dv", "do"):
            x, y = getattr(c, name).clone(), getattr(clean, name).clone()
            x[rows, col] = y[rows, col] = 0.0
            at = [(slice(0, 300), 3), (slice(301, 500), 1), (slice(500, 900), 2), (slice(900, 1200), 0)]
            for r, k in at:
                x[r, k] = y[r, k] = 0.0
            assert torch.equal(x, y), name
    assert bool(torch.isnan(c.y[100:300, 3]).all()) and bool(torch.isnan(c.y[310:500, 1]).all()) and bool(torch.isfinite(c.y[:100, 3]).all())
    assert bool(torch.isnan(c.dv[900:1001, 0]).all()) and bool(torch.isfinite(c.dv[1001:, 0]).all())


def test_states_may_be_updated_in_place_and_chunks_of_a_text_follow_one_another():
    c = Case(2000, 130, 4, seed=1)
    hp.hpsgd_gated_scan_forward(c.forward())
    state = c.h0.clone()
    hp.hpsgd_gated_scan_forward(c.forward(h0=state, h_last=state, y=torch.empty_like(c.y), ldy=130))
    assert torch.equal(state, c.h_last)
    # 500 rows a sequence: token by token (rows == sequences), against all at once
    state, f, v, o = c.h0.clone(), *(x.reshape(4, 500, 130) for x in (c.f, c.v, c.o))
    y = torch.empty(4, 500, 130, device="cuda")
    for t in range(500):
        step = torch.empty(4, 130, device="cuda")
        hp.hpsgd_gated_scan_forward(hp.make_gated_scan_forward(4, 130, 4, hp.HPSGD_F32, f[:, t].contiguous(), v[:, t].contiguous(), step, o=o[:, t].contiguous(), h0=state, h_last=state))
        y[:, t] = step
    torch.cuda.synchronize()
    want = ref.forward(*c.host())
    # both are within their bounds of the exact values
    got = y.reshape(2000, 130).double().cpu().numpy()
    assert (np.abs(got - want["y"]) <= want["y_err"] + 2.0 ** -24 * np.abs(want["y"])).all()
    assert (np.abs(state.double().cpu().numpy() - want["h_last"]) <= want["h_last_err"]).all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_gradients_may_take_the_inputs_memory(dtype):
    a, b = (Case(1500, 70, 3, bounds=[0, 333, 700, 1490], dtype=dtype, seed=2) for _ in range(2))
    hp.hpsgd_gated_scan_forward(a.forward())
    hp.hpsgd_gated_scan_backward(a.backward())
    hp.hpsgd_gated_scan_forward(b.forward())
    hp.hpsgd_gated_scan_backward(b.backward(df=b.f, dv=b.dy, do=b.v))
    torch.cuda.synchronize()
    for x, y in ((a.df, b.f), (a.dv, b.dy), (a.do, b.v)):
        assert torch.equal(x[:1490], y[:1490])


def test_the_same_bits_every_time_and_from_a_graph():
    c = Case(5000, 200, 7, bounds=[0, 5, 1200, 1200, 2500, 2600, 4000, 4999], dtype=BF, seed=4)
    calls = [(hp.hpsgd_gated_scan_forward, c.forward()), (hp.hpsgd_gated_scan_backward, c.backward())]
    outs = (c.y, c.h_last, c.df, c.dv, c.do, c.dh0)

    def run():
        for call, args in calls:
            call(args)

    run()
    first = [x.clone() for x in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    c.offsets.copy_(torch.tensor([0, 700, 700, 1800, 1801, 3000, 3000, 4990]))          # other sequences in the same graph
    graph.replay()
    other = [x.clone() for x in outs]
    run()
    assert all(torch.equal(x, y) for x, y in zip(other, outs))
    c.offsets.copy_(torch.tensor([0, 5, 1200, 1200, 2500, 2600, 4000, 4999]))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x[:4990], y[:4990]) for x, y in zip(first, outs))


def test_offsets_that_are_wrong_reach_nothing_outside():
    """Descending, negative and too large offsets: results are undefined, what lies around the call's memory is not touched."""
    for bad in ([900, 100, 500, 200, 0], [-50, 100, 1 << 40, 300, 2000], [0, 1 << 33, -(1 << 33), 5, 1000]):
        c = Case(1000, 66, 4, bounds=[0, 1, 2, 3, 1000], seed=6, pad=2)
        c.offsets.copy_(torch.tensor(bad))
        hp.hpsgd_gated_scan_forward(c.forward())
        hp.hpsgd_gated_scan_backward(c.backward())
        torch.cuda.synchronize()
        for x in (c.y, c.df, c.dv, c.do):
            assert float((x.as_strided((1000, 2), (68, 1), x.storage_offset() + 66) - MARK).abs().max()) == 0.0
            assert float((x._base[-8:] - MARK).abs().max()) == 0.0


def test_offsets_beyond_2_to_the_31_elements():
    rows, cols, tail = 70_000, 32_768, 300
    x = torch.zeros(rows, cols, dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    x[-tail:] = torch.randn(tail, cols, generator=g, device="cuda").to(BF)
    y, saved = torch.empty(rows, cols, dtype=BF, device="cuda"), torch.empty(hp.hpsgd_gated_scan_saved_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    hp.hpsgd_gated_scan_forward(hp.make_gated_scan_forward(rows, cols, 1, hp.HPSGD_BF16, x, x, y, saved=saved))
    df, dv = torch.empty_like(x), torch.empty_like(x)
    hp.hpsgd_gated_scan_backward(hp.make_gated_scan_backward(rows, cols, 1, hp.HPSGD_BF16, x, x, saved, x, df, dv))
    s = x[-tail:].clone()
    sy, ssaved = torch.empty_like(s), torch.empty(hp.hpsgd_gated_scan_saved_bytes(tail, cols), dtype=torch.uint8, device="cuda")
    sdf, sdv = torch.empty_like(s), torch.empty_like(s)
    hp.hpsgd_gated_scan_forward(hp.make_gated_scan_forward(tail, cols, 1, hp.HPSGD_BF16, s, s, sy, saved=ssaved))
    hp.hpsgd_gated_scan_backward(hp.make_gated_scan_backward(tail, cols, 1, hp.HPSGD_BF16, s, s, ssaved, s, sdf, sdv))
    # rows are grouped differently, so the last place of binary32 may differ, and with it a rounding to bf16: one step of 2^-7
    for a, b in ((y, sy), (df, sdf), (dv, sdv)):
        assert float((a[-tail:].float() - b.float()).abs().sub(b.float().abs() * 2.0 ** -7).max()) <= 1e-6
        assert float(a[: rows - tail - 200].abs().max()) == 0.0
