"""The recurrence, the loss and the gated layer: calls without a stream go to torch's current stream, and two at once on two streams do not disturb one another."""
import pytest
import torch

import paper_2009_02701_b200 as hp
from paper_2009_02701_b200 import binding
from tests.test_gpu_ops_streams import Recorder

pytestmark = pytest.mark.gpu

BF, U8 = torch.bfloat16, torch.uint8
ROWS, D, VOCAB = 96, 128, 1000


class Chain:
    """One call of each behind another: a recurrence's output through a gated layer to logits, the loss, and back."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        z = lambda *s, dtype=BF: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.fvo, self.w, self.out = rnd(ROWS, 3 * D).to(BF), rnd(2 * D, D) / 11.0, rnd(VOCAB, D) / 11.0
        self.y, self.saved, self.dfvo = z(ROWS, D), z(hp.hpsgd_gated_scan_saved_bytes(ROWS, D), dtype=U8), z(ROWS, 3 * D)
        self.labels = torch.randint(0, VOCAB, (ROWS,), generator=g, device="cuda")
        codes = lambda r, c: (z(r, -(-c // 16) * 16, dtype=U8), z(-(-c // 512), r, 4, dtype=U8))  # noqa: E731
        self.yq, self.wq, self.zq, self.oq, self.oqt, self.dlq = codes(ROWS, D), codes(2 * D, D), codes(ROWS, D), codes(VOCAB, D), codes(D, VOCAB), codes(ROWS, VOCAB)
        self.dq, self.dqt, self.wqt = codes(ROWS, 2 * D), codes(2 * D, ROWS), codes(D, 2 * D)
        self.gu, self.logits, self.dlogits, self.dz, self.dy, self.loss = z(ROWS, 2 * D), z(ROWS, VOCAB), z(ROWS, VOCAB), z(ROWS, D), z(ROWS, D), z(ROWS, dtype=torch.float32)
        side = dict(f=self.fvo[:, :D], v=self.fvo[:, D: 2 * D], o=self.fvo[:, 2 * D:], ldf=3 * D, ldv=3 * D, ldo=3 * D)
        q = lambda r, c, dt, x, a=None, b=None: (hp.hpsgd_quantize_fp8, hp.make_quantize_fp8(r, c, dt, x, q=a and a[0], scale=a and a[1], qt=b and b[0], scale_t=b and b[1]))  # noqa: E731
        gemm = lambda m, n, k, a, b, d: (hp.hpsgd_gemm_fp8, hp.make_gemm_fp8(m, n, k, *a, *b, d, hp.HPSGD_BF16, workspace=z(16 + hp.hpsgd_gemm_fp8_bytes(m, n, k), dtype=U8)))  # noqa: E731
        self.list = [
            (hp.hpsgd_gated_scan_forward, hp.make_gated_scan_forward(ROWS, D, 4, hp.HPSGD_BF16, y=self.y, saved=self.saved, **side)),
            q(ROWS, D, hp.HPSGD_BF16, self.y, self.yq), q(2 * D, D, hp.HPSGD_F32, self.w, self.wq, self.wqt), q(VOCAB, D, hp.HPSGD_F32, self.out, self.oq, self.oqt),
            (hp.hpsgd_gated_ffn_forward, hp.make_gated_ffn_forward(ROWS, D, D, hp.HPSGD_SILU, *self.yq, *self.wq, z8=self.zq[0], z_scale=self.zq[1], gu=self.gu)),
            gemm(ROWS, VOCAB, D, self.zq, self.oq, self.logits),
            (hp.hpsgd_distill_loss, hp.make_distill_loss(ROWS, VOCAB, 0, hp.HPSGD_BF16, self.logits, labels=self.labels, loss=self.loss, dlogits=self.dlogits, grad_scale=1.0 / ROWS)),
            q(ROWS, VOCAB, hp.HPSGD_BF16, self.dlogits, self.dlq),
            gemm(ROWS, D, VOCAB, self.dlq, self.oqt, self.dz),
            (hp.hpsgd_gated_ffn_backward, hp.make_gated_ffn_backward(ROWS, D, hp.HPSGD_SILU, self.gu, self.dz, hp.HPSGD_BF16, dq=self.dq[0], dq_scale=self.dq[1], dqt=self.dqt[0], dqt_scale=self.dqt[1])),
            gemm(ROWS, D, 2 * D, self.dq, self.wqt, self.dy),
            (hp.hpsgd_gated_scan_backward, hp.make_gated_scan_backward(ROWS, D, 4, hp.HPSGD_BF16, saved=self.saved, dy=self.dy, df=self.dfvo[:, :D], dv=self.dfvo[:, D: 2 * D],
                                                                       do=self.dfvo[:, 2 * D:], lddf=3 * D, lddv=3 * D, lddo=3 * D, **side)),
        ]

    def run(self, **kw):
        for call, args in self.list:
            call(args, **kw)

    def results(self):
        return [x.clone() for x in (self.loss, self.dlogits, self.dy, self.dfvo)]


def test_the_stream_that_a_call_goes_to(monkeypatch):
    c, side, other, fake = Chain(0), torch.cuda.Stream(), torch.cuda.Stream(), Recorder()
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_lib", fake)
    for where, kw, want in ((torch.cuda.default_stream(), {}, 0), (side, {}, side.cuda_stream), (side, dict(stream=other), other.cuda_stream), (side, dict(stream=0), 0)):
        fake.streams.clear()
        with torch.cuda.stream(where):
            c.run(**kw)
        assert fake.streams == [want] * len(c.list)


def test_a_chain_of_them_on_two_streams_at_once_and_from_a_graph():
    chains = [Chain(k) for k in (1, 2)]
    want = []
    for c in chains:
        c.run()
        want.append(c.results())
    hp.hpsgd_ops_check()
    assert all(bool(torch.isfinite(x.float()).all()) and float(x.float().abs().max()) > 0 for w in want for x in w)
    streams = [torch.cuda.Stream() for _ in chains]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(chains, streams):
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c, w in zip(chains, want):
        assert all(torch.equal(x, y) for x, y in zip(c.results(), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chains[0].run()
    chains[0].fvo.copy_(chains[1].fvo)
    for name in ("w", "out", "labels"):
        getattr(chains[0], name).copy_(getattr(chains[1], name))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(chains[0].results(), want[1]))
    hp.hpsgd_ops_check()
