"""A small language model trained by K simulated workers: 8-bit layers forward and backward, AdamW with 8-bit moments on each
worker's replica, the delayed merge of HPSGD between rounds.

    python examples/train_lm.py [--rounds 40] [--workers 4] [--bits 8]

The model: token embedding, two blocks (norm, linear to 4 d, squared ReLU, linear back, residual), final norm, output projection.  Every
linear layer runs in the 8-bit block format (forward, input gradient, weight gradient); norms take the residual's addition and hand
their output over in 8 bits.  The embedding's look-up, the activation and the cross-entropy are torch's.  The text is synthetic: a Markov chain
over the vocabulary in which each token has a few likely successors, so the loss can fall from log(vocabulary) to the chain's entropy.
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

    def __init__(self, vocab, d, blocks, tokens):
        self.vocab, self.d, self.blocks, self.tokens = vocab, d, blocks, tokens
        self.shapes = [("embed", (vocab, d))]
        for b in range(blocks):
            self.shapes += [("norm%d" % b, (d,)), ("up%d" % b, (4 * d, d)), ("down%d" % b, (d, 4 * d))]
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

    # ---- the model
    def loss_and_gradients(self, p, g, tokens, targets):
        """p, g: the views of parameters and gradients.  Returns the loss as a device scalar; g is overwritten."""
        x, residual, saved = p["embed"][tokens].to(BF), None, []
        for b in range(self.blocks):
            y, h, n = self.norm(x, p["norm%d" % b], residual)
            z, l1 = self.linear(y, p["up%d" % b])
            r = torch.relu(z)
            a, _ = self.quantize(r * r, hp.HPSGD_BF16, transposed=False)
            x, l2 = self.linear(a, p["down%d" % b])
            residual = h
            saved.append((n, l1, r, l2))
        y, h, last = self.norm(x, p["norm"], residual)
        logits, lo = self.linear(y, p["out"])
        logp = torch.log_softmax(logits.float(), dim=1)
        loss = -logp.gather(1, targets[:, None]).mean()
        d = torch.exp(logp)
        d.scatter_add_(1, targets[:, None], torch.full_like(d[:, :1], -1.0))
        dy = self.linear_backward(lo, (d / len(targets)).to(BF), g["out"])
        dh = self.norm_backward(last, dy, None, g["norm"])
        for b in reversed(range(self.blocks)):
            n, l1, r, l2 = saved[b]
            da = self.linear_backward(l2, dh, g["down%d" % b])
            dz = da * 2 * r
            dy = self.linear_backward(l1, dz, g["up%d" % b])
            dh = self.norm_backward(n, dy, dh, g["norm%d" % b])
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


def train(rounds=40, workers=4, bits=8, vocab=512, d=256, blocks=2, tokens=2048, lr=3e-3, staleness=1, out=print):
    """Returns the mean loss of the workers in each round."""
    model, chain = Model(vocab, d, blocks, tokens), Chain(vocab)
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

        def replica(i):          # the worker's replica inside the lent arena; complete behind the merge that cloned it
            hp.hpsgd_synchronize()
            at = hp.hpsgd_get_replica(i)[0] - arena.data_ptr()
            return arena[at: at + 4 * P_pad].view(F32)

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
                    batch = chain.batch(tokens, 1000 * t + i)
                    losses.append(model.loss_and_gradients(model.views(replica(i)), model.views(grads[i]), *batch))
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
    a = ap.parse_args()
    print("uniform guessing: %.3f, the chain's entropy: %.3f" % (math.log(512), -sum(p * math.log(p) for p in (0.5, 0.25, 0.15, 0.1))))
    train(a.rounds, a.workers, a.bits)
