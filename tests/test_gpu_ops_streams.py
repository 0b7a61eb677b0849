"""The operators' calls without a stream go to torch's current stream; with one, to that one."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from paper_2009_02701_b200 import binding

pytestmark = pytest.mark.gpu

U8, BF = torch.uint8, torch.bfloat16
ROWS, COLS = 64, 256


class Buffers:
    """One small call of each kind and its buffers."""

    def __init__(self):
        z = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.x, self.w, self.rstd = z(ROWS, COLS), z(COLS), z(ROWS)
        self.q, self.s = z(ROWS, COLS, dtype=U8), z(1, ROWS, 4, dtype=U8)
        self.y, self.dx, self.dw, self.d = z(ROWS, COLS), z(ROWS, COLS), z(COLS), z(ROWS, ROWS)
        self.ws, self.norm = z(max(hp.HPSGD_GRAD_NORM_WORKSPACE, hp.hpsgd_rmsnorm_backward_bytes(ROWS, COLS)), dtype=U8), z(2)
        self.m, self.v, self.p = z(ROWS * COLS), z(ROWS * COLS), z(ROWS * COLS)
        self.table = hp.make_adamw_table([dict(param=self.p, grad=self.x, m=self.m, v=self.v, n=ROWS * COLS)], 0, 0, 32)
        self.forward = hp.make_rmsnorm_forward(ROWS, COLS, 1e-5, 0, self.x, self.w, y=self.y, rstd=self.rstd)
        self.backward = hp.make_rmsnorm_backward(ROWS, COLS, 0, self.x, self.w, self.rstd, self.y, self.dx, self.dw, self.ws)
        self.quantize = hp.make_quantize_fp8(ROWS, COLS, 0, self.x, q=self.q, scale=self.s)
        self.product = hp.make_gemm_fp8(ROWS, ROWS, COLS, self.q, self.s, self.q, self.s, self.d, 0)

    def calls(self, **kw):
        hp.hpsgd_grad_norm(self.table, 1.0, self.ws, self.norm, **kw)
        hp.hpsgd_adamw_step(self.table, 1e-3, 0.9, 0.999, 1e-8, 1, grad_scale=self.norm[1:], **kw)
        hp.hpsgd_rmsnorm_forward(self.forward, **kw)
        hp.hpsgd_rmsnorm_backward(self.backward, **kw)
        hp.hpsgd_quantize_fp8(self.quantize, **kw)
        hp.hpsgd_gemm_fp8(self.product, **kw)


class Recorder:
    """Stands in for the library: notes the stream, which every call has as its last argument."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            self.streams.append(args[-1] or 0)
            return 0
        return call


def test_the_stream_that_a_call_goes_to(monkeypatch):
    b, side, other, fake = Buffers(), torch.cuda.Stream(), torch.cuda.Stream(), Recorder()
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_lib", fake)
    for where, kw, want in ((torch.cuda.default_stream(), {}, 0), (side, {}, side.cuda_stream), (side, dict(stream=other), other.cuda_stream),
                            (side, dict(stream=0), 0), (side, dict(stream=other.cuda_stream), other.cuda_stream)):
        fake.streams.clear()
        with torch.cuda.stream(where):
            b.calls(**kw)
            hp.hpsgd_ops_check(**kw)
        assert fake.streams == [want] * 7


def test_work_without_a_stream_is_ordered_with_torch_s():
    """On a stream of torch's own pool, which the legacy default stream does not wait for: the input is ready behind 100 large products."""
    side = torch.cuda.Stream()
    b = Buffers()
    big = torch.randn(4096, 4096, device="cuda").to(BF)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(100):
            big = (big @ big).clamp(-1.0, 1.0)
        b.x.fill_(2.0)
        hp.hpsgd_quantize_fp8(b.quantize)
        out = b.q.clone()
    side.synchronize()
    assert bool((out == 0x78).all())           # 2 = 256 * 2^-7, the smallest scale with 448 * 2^e >= 2


def test_calls_without_a_stream_are_captured():
    b = Buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.calls()
    b.x.fill_(1.0)
    b.w.fill_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    assert abs(float(b.norm[0]) - 128.0) < 1e-3 and float(b.y[3, 7]) == pytest.approx(1.0, rel=1e-4) and float(b.d[5, 6]) == 256.0
