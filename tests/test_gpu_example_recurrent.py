"""The example with the recurrence, the gated layer and the teacher: that it runs, that a run repeats, and its gradients."""
import math

import pytest
import torch

from examples import train_lm

pytestmark = pytest.mark.gpu

SMALL = dict(vocab=128, d=128, blocks=1, tokens=256, sequences=4, out=lambda s: None)


@pytest.mark.parametrize("options", [dict(recurrent=True), dict(gated=True), dict(distil=0.5), dict(recurrent=True, gated=True, distil=0.3)], ids=str)
def test_it_runs_and_a_run_repeats_bit_for_bit(options):
    a, b = (train_lm.train(rounds=3, workers=2, **SMALL, **options) for _ in range(2))
    assert a == b and len(a) == 3 and all(math.isfinite(x) for x in a)


def plain(model, p, tokens, targets, teacher, share):
    """The same model in binary32 torch operations, with nothing rounded to fewer bits."""
    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-5) * w

    d, x = model.d, p["embed"][tokens]
    for b in range(model.blocks):
        if model.recurrent:
            z = norm(x, p["mixnorm%d" % b]) @ p["mix%d" % b].t()
            a, v = torch.sigmoid(z[:, :d]), z[:, d: 2 * d]
            a, v = (t.reshape(model.sequences, -1, d) for t in (a, v))
            h, rows = torch.zeros(model.sequences, d, device="cuda"), []
            for t in range(a.shape[1]):
                h = a[:, t] * h + (1 - a[:, t]) * v[:, t]
                rows.append(h)
            x = x + (torch.stack(rows, dim=1).reshape(-1, d) * torch.sigmoid(z[:, 2 * d:])) @ p["mixout%d" % b].t()
        z = norm(x, p["norm%d" % b]) @ p["up%d" % b].t()
        n = z.shape[1] // 2
        x = x + (torch.nn.functional.silu(z[:, :n]) * z[:, n:] if model.gated else torch.relu(z).square()) @ p["down%d" % b].t()
    logits = norm(x, p["norm"]) @ p["out"].t()
    loss = (1 - share) * torch.nn.functional.cross_entropy(logits, targets)
    if teacher is not None:
        values, index = teacher.float().topk(8, dim=1)
        t = torch.softmax(values / 2.0, dim=1)
        q = torch.log_softmax(logits / 2.0, dim=1).gather(1, index)
        loss = loss + share * 4.0 * (t * (t.log() - q)).sum(dim=1).mean()
    return loss


@pytest.mark.parametrize("options,share", [(dict(recurrent=True), 0.0), (dict(gated=True), 0.0), (dict(recurrent=True, gated=True), 0.4)], ids=str)
def test_gradients_against_autograd(options, share):
    """Every parameter's gradient, against that of the same model in binary32.  A value rounded to an E4M3 code is off by at most 2^-4 of itself, 0.036 in the
    mean square; on the way to a gradient lie at most 2 operands x 6 linear layers x 2 directions of them, in quadrature 0.18, doubled for what the
    layers between make of it: the cosine of two gradients is then above sqrt(1 - 0.36^2) = 0.93 and their lengths are within 0.36.  The loss: a mean over
    256 rows of logits that are off by 0.36 of about 1 each."""
    model = train_lm.Model(128, 128, 1, 256, 4, **options)
    chain, gen = train_lm.Chain(128), torch.Generator().manual_seed(5)
    flat = torch.cat([torch.nn.functional.pad((torch.ones(s) if len(s) == 1 else torch.randn(*s, generator=gen) * (1.0 if n == "embed" else 1.0 / math.sqrt(s[1]))).view(-1), (0, 0))
                      for n, s in model.shapes])
    room = torch.zeros(train_lm.hp.hpsgd_layout_padded(model.sizes)[0], device="cuda")
    grads = torch.zeros_like(room)
    at = 0
    for o, k in zip(model.offsets, model.sizes):
        room[o: o + k] = flat[at: at + k].cuda()
        at += k
    tokens, targets = chain.text(4, 64, 9)
    teacher = torch.randn(256, 128, generator=gen).cuda().to(torch.bfloat16) * 3.0 if share else None
    loss = model.loss_and_gradients(model.views(room), model.views(grads), tokens, targets, teacher=teacher, share=share)
    p = {n: v.clone().requires_grad_(True) for n, v in model.views(room).items()}
    want = plain(model, p, tokens, targets, teacher, share)
    want.backward()
    assert abs(float(loss) - float(want)) < 0.36
    for name, g in model.views(grads).items():
        a, b = g.double().view(-1), p[name].grad.double().view(-1)
        cosine = float((a @ b) / (a.norm() * b.norm()))
        assert cosine > 0.93 and abs(float(a.norm() / b.norm()) - 1.0) < 0.36, (name, cosine, float(a.norm() / b.norm()))
