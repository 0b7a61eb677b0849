"""A small language model trained by K simulated workers: 8-bit layers forward and backward, AdamW with 8-bit moments on each
worker's replica, the delayed merge of HPSGD between rounds.

    python examples/train_lm.py [--rounds 40] [--workers 4] [--bits 8] [--recurrent] [--gated] [--distil 0.3]

The model: token embedding, two blocks (norm, linear to 4 d, squared ReLU, linear back, residual), final norm, output projection.  Every
linear layer runs in the 8-bit block format (forward, input gradient, weight gradient); norms take the residual's addition and hand
their output over in 8 bits.  The embedding's look-up, the activation and the cross-entropy are torch's.  The text is synthetic: a Markov chain
over the vocabulary in which each token has a few likely successors, so the loss can fall from log(vocabulary) to the chain's entropy.

With --recurrent each block begins with a gated linear recurrence over the sequences of the batch (norm, one linear to gates, values and output gates,
the recurrence, linear back, residual); with --gated the linear to 4 d is a gated one (two projections, SiLU and product in one kernel); with
--distil the workers learn a part of their loss from the eight top logits that the model they share, the one that the merge commits, gives for
their batch.  Loss and gradient are then the library's too.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2009_02701_b200 as hp  # noqa: E402

BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def up(n, a):
    return -(-n // a) * a


class Codes:
    """Room for a matrix [rows, cols] in the 8-bit block format."""

    def __init__(self, rows, cols):
        self.rows, self.cols = rows, cols
        self.q = torch.zeros(rows, up(cols, 16), dtype=U8, device="cuda")
        self.s = torch.zeros(up(up(cols, 128) // 128, 4) // 4, rows, 4, dtype=U8, device="cuda")


class Model:
    """Shapes, buffers and the passes; the parameters come in as one flat fp32 tensor (a worker's replica) and the gradients go out as one."""

    def __init__(self, vocab, d, blocks, tokens, sequences=1, recurrent=False, gated=False):
        self.vocab, self.d, self.blocks, self.tokens = vocab, d, blocks, tokens
        self.sequences, self.recurrent, self.gated = sequences, recurrent, gated
        self.shapes = [("embed", (vocab, d))]
        for b in range(blocks):
            if recurrent:
                self.shapes += [("mixnorm%d" % b, (d,)), ("mix%d" % b, (3 * d, d)), ("mixout%d" % b, (d, d))]
            self.shapes += [("norm%d" % b, (d,)), ("up%d" % b, ((8 if gated else 4) * d, d)), ("down%d" % b, (d, 4 * d))]
        self.shapes += [("norm", (d,)), ("out", (vocab, d))]
        self.sizes = [math.prod(s) for _, s in self.shapes]
        _, self.offsets = hp.hpsgd_layout_padded(self.sizes)
        self.workspaces = {}

    def views(self, flat):
        return {n: flat[o:o + k].view(s) for (n, s), o, k in zip(self.shapes, self.offsets, self.sizes)}

    def stream(self):
        return torch.cuda.current_stream()

    # ---- layers
    def quantize(self, x, dtype, rows=True, transposed=True):
        r, c = x.shape
        a, b = Codes(r, c) if rows else None, Codes(c, r) if transposed else None
        hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(r, c, dtype, x, q=a and a.q, scale=a and a.s, qt=b and b.q, scale_t=b and b.s), self.stream())
        return a, b

    def transpose(self, x):
        t = Codes(x.cols, x.rows)
        hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(x.rows, x.cols, hp.HPSGD_FP8, x.q, x_scale=x.s, qt=t.q, scale_t=t.s), self.stream())
        return t

    def product(self, a, b, out):
        """out [a.rows, b.rows] = a b^T"""
        key = (a.rows, b.rows, a.cols)
        if key not in self.workspaces:
            self.workspaces[key] = torch.zeros(max(16, hp.hpsgd_gemm_fp8_bytes(*key)), dtype=U8, device="cuda")
        hp.hpsgd_gemm_fp8(hp.make_gemm_fp8(*key, a.q, a.s, b.q, b.s, out, hp.HPSGD_F32 if out.dtype == F32 else hp.HPSGD_BF16,
                                           workspace=self.workspaces[key]), self.stream())
        return out

    def new(self, *shape, dtype=BF):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def linear(self, x, w):
        """x in the block format, w fp32 [N, K] -> y bf16, and what the backward pass needs."""
        wq, wt = self.quantize(w, hp.HPSGD_F32)
        return self.product(x, wq, self.new(x.rows, wq.rows)), (x, wt)

    def linear_backward(self, saved, dy, dw):
        """dy bf16 -> dx bf16; the weight's gradient to dw."""
        x, wt = saved
        g, gt = self.quantize(dy, hp.HPSGD_BF16)
        self.product(gt, self.transpose(x), dw)
        return self.product(g, wt, self.new(g.rows, wt.rows))

    def norm(self, x, weight, residual=None):
        rows, cols = x.shape
        h, y, rstd = (self.new(rows, cols) if residual is not None else x), Codes(rows, cols), self.new(rows, dtype=F32)
        hp.hpsgd_rmsnorm_forward(hp.make_rmsnorm_forward(rows, cols, 1e-5, hp.HPSGD_BF16, x, weight, residual=residual, h=h if residual is not None else None,
                                                         y8=y.q, y_scale=y.s, rstd=rstd, weight_dtype=hp.HPSGD_F32), self.stream())
        return y, h, (h, weight, rstd)

    def norm_backward(self, saved, dy, dres, dweight):
        h, weight, rstd = saved
        rows, cols = h.shape
        ws = self.new(hp.hpsgd_rmsnorm_backward_bytes(rows, cols), dtype=U8)
        dx = self.new(rows, cols)
        hp.hpsgd_rmsnorm_backward(hp.make_rmsnorm_backward(rows, cols, hp.HPSGD_BF16, h, weight, rstd, dy, dx, dweight, ws, dres=dres,
                                                           weight_dtype=hp.HPSGD_F32), self.stream())
        return dx

    def scan(self, z):
        """z bf16 [tokens, 3 d]: gates, values and output gates of sequences that follow one another -> bf16 [tokens, d], and what the backward pass needs."""
        rows, d = z.shape[0], self.d
        y, kept = self.new(rows, d), self.new(hp.hpsgd_gated_scan_saved_bytes(rows, d), dtype=U8)
        side = dict(f=z[:, :d], v=z[:, d: 2 * d], o=z[:, 2 * d:], ldf=3 * d, ldv=3 * d, ldo=3 * d)
        hp.hpsgd_gated_scan_forward(hp.make_gated_scan_forward(rows, d, self.sequences, hp.HPSGD_BF16, y=y, saved=kept, **side), self.stream())
        return y, (side, kept)

    def scan_backward(self, saved, dy):
        side, kept = saved
        rows, d = dy.shape
        dz = self.new(rows, 3 * d)
        hp.hpsgd_gated_scan_backward(hp.make_gated_scan_backward(rows, d, self.sequences, hp.HPSGD_BF16, saved=kept, dy=dy, df=dz[:, :d], dv=dz[:, d: 2 * d],
                                                                 do=dz[:, 2 * d:], lddf=3 * d, lddv=3 * d, lddo=3 * d, **side), self.stream())
        return dz

    def gated_linear(self, x, w):
        """x in the block format, w fp32 [2 N, K] -> silu(x w_gate^T) * (x w_up^T) in the block format, and what the backward pass needs."""
        wq, wt = self.quantize(w, hp.HPSGD_F32)
        n = wq.rows // 2
        z, gu = Codes(x.rows, n), self.new(x.rows, 2 * n)
        hp.hpsgd_gated_ffn_forward(hp.make_gated_ffn_forward(x.rows, n, x.cols, hp.HPSGD_SILU, x.q, x.s, wq.q, wq.s, z8=z.q, z_scale=z.s, gu=gu), self.stream())
        return z, (x, wt, gu)

    def gated_linear_backward(self, saved, dz, dw):
        """dz bf16 -> dx bf16; the weight's gradient to dw."""
        x, wt, gu = saved
        rows, n = dz.shape
        g, gt = Codes(rows, 2 * n), Codes(2 * n, rows)
        hp.hpsgd_gated_ffn_backward(hp.make_gated_ffn_backward(rows, n, hp.HPSGD_SILU, gu, dz, hp.HPSGD_BF16, dq=g.q, dq_scale=g.s, dqt=gt.q, dqt_scale=gt.s), self.stream())
        self.product(gt, self.transpose(x), dw)
        return self.product(g, wt, self.new(rows, wt.rows))

    def loss(self, logits, targets, teacher=None, share=0.0, temperature=2.0):
        """Mean loss as a device scalar, and its gradient bf16.  teacher: logits of which the eight largest are learnt from, with a share of the loss."""
        rows, vocab = logits.shape
        each, d, top = self.new(rows, dtype=F32), self.new(rows, vocab), {}
        if teacher is not None:
            values, index = teacher.topk(8, dim=1)
            top = dict(teacher_index=index.int(), teacher_logits=values.contiguous(), teacher_weight=share, temperature=temperature)
        hp.hpsgd_distill_loss(hp.make_distill_loss(rows, vocab, 8 if top else 0, hp.HPSGD_BF16, logits, labels=targets, label_weight=1.0 - share, loss=each, dlogits=d,
                                                   grad_scale=1.0 / rows, **top), self.stream())
        return each.mean(), d

    # ---- the model
    def forward(self, p, tokens):
        """Logits bf16, and what the backward pass needs."""
        x, residual, saved = p["embed"][tokens].to(BF), None, []
        for b in range(self.blocks):
            mix = None
            if self.recurrent:
                y, residual, n = self.norm(x, p["mixnorm%d" % b], residual)
                z, l1 = self.linear(y, p["mix%d" % b])
                r, s = self.scan(z)
                x, l2 = self.linear(self.quantize(r, hp.HPSGD_BF16, transposed=False)[0], p["mixout%d" % b])
                mix = (n, l1, s, l2)
            y, residual, n = self.norm(x, p["norm%d" % b], residual)
            if self.gated:
                a, l1 = self.gated_linear(y, p["up%d" % b])
                r = None
            else:
                z, l1 = self.linear(y, p["up%d" % b])
                r = torch.relu(z)
                a, _ = self.quantize(r * r, hp.HPSGD_BF16, transposed=False)
            x, l2 = self.linear(a, p["down%d" % b])
            saved.append((mix, n, l1, r, l2))
        y, _, last = self.norm(x, p["norm"], residual)
        logits, lo = self.linear(y, p["out"])
        return logits, (saved, last, lo)

    def loss_and_gradients(self, p, g, tokens, targets, teacher=None, share=0.0):
        """p, g: the views of parameters and gradients.  Returns the loss as a device scalar; g is overwritten."""
        logits, (saved, last, lo) = self.forward(p, tokens)
        if self.recurrent or self.gated or teacher is not None:
            loss, d = self.loss(logits, targets, teacher, share)
        else:
            logp = torch.log_softmax(logits.float(), dim=1)
            loss = -logp.gather(1, targets[:, None]).mean()
            d = torch.exp(logp)
            d.scatter_add_(1, targets[:, None], torch.full_like(d[:, :1], -1.0))
            d = (d / len(targets)).to(BF)
        dy = self.linear_backward(lo, d, g["out"])
        dh = self.norm_backward(last, dy, None, g["norm"])
        for b in reversed(range(self.blocks)):
            mix, n, l1, r, l2 = saved[b]
            da = self.linear_backward(l2, dh, g["down%d" % b])
            if self.gated:
                dy = self.gated_linear_backward(l1, da, g["up%d" % b])
            else:
                dz = da * 2 * r
                dy = self.linear_backward(l1, dz, g["up%d" % b])
            dh = self.norm_backward(n, dy, dh, g["norm%d" % b])
            if mix is not None:
                n, l1, s, l2 = mix
                dz = self.scan_backward(s, self.linear_backward(l2, dh, g["mixout%d" % b]))
                dh = self.norm_backward(n, self.linear_backward(l1, dz, g["mix%d" % b]), dh, g["mixnorm%d" % b])
        g["embed"].zero_().index_put_((tokens,), dh.float(), accumulate=True)      # (sorted: the same sum every time)
        return loss


class Chain:
    """Each token is followed by one of four successors with probabilities 0.5, 0.25, 0.15, 0.1: entropy 1.21 nats."""

    def __init__(self, vocab, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.next = torch.randint(0, vocab, (vocab, 4), generator=g).cuda()
        self.p = torch.tensor([0.5, 0.25, 0.15, 0.1], device="cuda")

    def batch(self, n, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        tokens = torch.randint(0, len(self.next), (n,), generator=g, device="cuda")
        return tokens, self.next[tokens, torch.multinomial(self.p, n, replacement=True, generator=g)]

    def text(self, sequences, length, seed):
        """The same from sequences that the chain itself writes, one behind another."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        words = [torch.randint(0, len(self.next), (sequences,), generator=g, device="cuda")]
        for _ in range(length):
            words.append(self.next[words[-1], torch.multinomial(self.p, sequences, replacement=True, generator=g)])
        x = torch.stack(words, dim=1)
        return x[:, :-1].reshape(-1), x[:, 1:].reshape(-1)


def train(rounds=40, workers=4, bits=8, vocab=512, d=256, blocks=2, tokens=2048, lr=3e-3, staleness=1, out=print, recurrent=False, gated=False, distil=0.0,
          sequences=16):
    """Returns the mean loss of the workers in each round."""
    model, chain = Model(vocab, d, blocks, tokens, sequences, recurrent, gated), Chain(vocab)
    hp.hpsgd_destroy()
    hp.hpsgd_set_layout(model.sizes)
    P_pad = hp.hpsgd_layout_padded(model.sizes)[0]
    # The arena and the main stream are lent, so that the workers' passes read their replicas and are ordered with the steps.
    arena = torch.zeros(hp.hpsgd_arena_bytes(P_pad, workers), dtype=U8, device="cuda")
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    hp.hpsgd_bind(arena, arena.numel(), main, side)
    hp.hpsgd_init(sum(model.sizes), workers, lr, 0.0, 1)
    try:
        hp.hpsgd_set_option(hp.HPSGD_OPT_STALENESS, staleness)
        g = torch.Generator().manual_seed(1)
        start = [torch.ones(s) if len(s) == 1 else torch.randn(*s, generator=g) * (1.0 if n == "embed" else 1.0 / math.sqrt(s[1])) for n, s in model.shapes]
        hp.hpsgd_set_global_host(torch.cat([x.view(-1) for x in start]).numpy())

        def inside(address):     # parameters inside the lent arena
            at = address - arena.data_ptr()
            return arena[at: at + 4 * P_pad].view(F32)

        def replica(i):          # the worker's replica; complete behind the merge that cloned it
            hp.hpsgd_synchronize()
            return inside(hp.hpsgd_get_replica(i)[0])

        dt = F32 if bits == 32 else U8
        moments = [[torch.zeros(P_pad, dtype=dt, device="cuda") for _ in range(2)] for _ in range(workers)]
        scales = [[torch.zeros(-(-P_pad // 128), dtype=U8, device="cuda") if bits == 8 else None for _ in range(2)] for _ in range(workers)]
        grads = [torch.zeros(P_pad, device="cuda") for _ in range(workers)]
        norm, ws = torch.zeros(2, device="cuda"), torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8, device="cuda")
        torch.cuda.synchronize()
        history = []
        with torch.cuda.stream(main):
            for t in range(rounds):
                rate = lr * min(1.0, (t + 1) / 5)
                losses = []
                for i in range(workers):
                    batch = chain.text(sequences, tokens // sequences, 1000 * t + i) if recurrent else chain.batch(tokens, 1000 * t + i)
                    mine, teacher = model.views(replica(i)), None
                    if distil:
                        teacher, _ = model.forward(model.views(inside(hp.hpsgd_get_global())), batch[0])
                    losses.append(model.loss_and_gradients(mine, model.views(grads[i]), *batch, teacher=teacher, share=distil))
                    table = hp.make_adamw_table([dict(grad=grads[i], n=P_pad)], hp.HPSGD_F32, hp.HPSGD_F32, bits)
                    hp.hpsgd_grad_norm(table, 1.0, ws, norm, main)
                    hp.hpsgd_local_step_adamw(i, grads[i], *moments[i], t + 1, rate, 0.9, 0.98, 1e-8, 0.01, bits, *scales[i], grad_scale=norm[1:])
                hp.hpsgd_sync_merge()
                history.append(float(torch.stack(losses).mean()))
                if t % 5 == 0 or t == rounds - 1:
                    out("round %3d  loss %.3f  gradient norm %.3f" % (t, history[-1], float(norm[0])))
        hp.hpsgd_synchronize()
        hp.hpsgd_ops_check(main)
    finally:
        hp.hpsgd_destroy()
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--recurrent", action="store_true")
    ap.add_argument("--gated", action="store_true")
    ap.add_argument("--distil", type=float, default=0.0)
    a = ap.parse_args()
    print("uniform guessing: %.3f, the chain's entropy: %.3f" % (math.log(512), -sum(p * math.log(p) for p in (0.5, 0.25, 0.15, 0.1))))
    train(a.rounds, a.workers, a.bits, recurrent=a.recurrent, gated=a.gated, distil=a.distil)
