"""Cases for measuring the operators of a recurrent language model: a gated linear recurrence over sequences (with its
gradients and its form for single tokens), a gated feed-forward layer in the 8-bit block format (with its gradients), and
the loss over labels and a teacher's top logits (with its gradient).

``run`` computes them in elementary torch operations where ``own`` is false, and through the package's entry
points where it is true.  ``exact`` restates their definitions in 64 bits.

Recurrence, per channel:  a = sigmoid(f),  h_t = a_t h_(t-1) + (1 - a_t) v_t,  y_t = h_t sigmoid(o_t).
Feed-forward:  g, u = x Wg^T, x Wu^T;  z = act(g) u.
Loss of a row:  wl (lse(z) - z[label]) + wt T^2 KL(p || softmax(z / T)),  p the softmax of the teacher's k logits / T.

The 8-bit block format: a matrix [rows, cols] is held as E4M3 codes and one power of two (E8M0) for every 128
consecutive columns of a row, the smallest 2^e >= 2^-127 with 448 * 2^e >= the block's largest magnitude.  Codes
are [rows, cols up to a multiple of 16]; the scale of block b of row r is entry [b // 4, r, b % 4] of an array
[ceil(blocks / 4), rows, 4].
"""
import math

import torch

own = False

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BF = torch.bfloat16
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GELU_1, GELU_3 = math.sqrt(2.0 / math.pi), 0.044715


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # generation: one token of each of 64 sequences, the states in and out (latency)
        dict(name="scan 64 tokens of 64 sequences", op="scan", train=False, rows=64, cols=1024, sequences=64, ragged=False, dtype="bf16", gate=True, states=True),
        # a long text read at once, its last state kept for what follows
        dict(name="scan 65536 tokens of one sequence", op="scan", train=False, rows=65536, cols=1024, sequences=1, ragged=False, dtype="bf16", gate=True, states=True),
        # a training step over a batch of equal sequences, forward and backward
        dict(name="scan train 16 x 1024", op="scan", train=True, rows=16384, cols=2048, sequences=16, ragged=False, dtype="bf16", gate=True, states=False),
        # the same in 32 bits over a packed batch of uneven sequences with room behind the last one
        dict(name="scan train ragged", op="scan", train=True, rows=8191, cols=1000, sequences=37, ragged=True, dtype="f32", gate=False, states=True),
        # a few rows of a small vocabulary (latency)
        dict(name="loss 8 x 512", op="loss", rows=8, vocab=512, k=8, temperature=2.0, dtype="bf16", labels=True, grad="with"),
        # a training step's loss over 30000 words: labels and a teacher's 64 top logits
        dict(name="loss 4096 x 30000", op="loss", rows=4096, vocab=30000, k=64, temperature=2.0, dtype="bf16", labels=True, grad="with"),
        # a large vocabulary, whose rows are more than one SM holds; temperature 1
        dict(name="loss 4096 x 131072", op="loss", rows=4096, vocab=131072, k=32, temperature=1.0, dtype="bf16", labels=True, grad="with"),
        # the gradient on its own, in 32 bits, rows off every boundary, the teacher alone
        dict(name="loss backward 2047 x 30011", op="loss", rows=2047, vocab=30011, k=17, temperature=3.0, dtype="f32", labels=False, grad="later"),
        # generation: one token through both projections
        dict(name="ffn 1 token", op="ffn", train=False, M=1, N=4096, K=1024, act="silu"),
        # a batch of prompts
        dict(name="ffn 8192 tokens", op="ffn", train=False, M=8192, N=8192, K=2048, act="silu"),
        # a training step's forward and backward, up to what the products for the gradients take
        dict(name="ffn train 4096 tokens", op="ffn", train=True, M=4096, N=4096, K=1024, act="gelu"),
        # sizes that no tile divides
        dict(name="ffn train ragged", op="ffn", train=True, M=1001, N=2744, K=1000, act="silu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan", "loss", "ffn"])
    if op == "scan":
        train = rng.random() < 0.6
        cols = _log(rng, 48, 4096)
        if rng.random() < 0.7:
            cols = _up(cols, 8)
        rows = _log(rng, 16 if train else 1, min(65536, 32 * 1024 * 1024 // cols))
        sequences = _log(rng, 1, min(rows, 512))
        ragged = rng.random() < 0.6
        if not ragged:
            rows = max(1, rows // sequences) * sequences
        return dict(op=op, train=train, rows=rows, cols=cols, sequences=sequences, ragged=ragged, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    gate=rng.random() < 0.6, states=rng.random() < 0.6)
    if op == "loss":
        vocab = _log(rng, 100, 131072)
        if rng.random() < 0.6:
            vocab = _up(vocab, 8)
        k = rng.choice([0, 1, 8, 50, 128])
        return dict(op=op, rows=_log(rng, 1, min(8192, 2 ** 28 // vocab)), vocab=vocab, k=min(k, vocab), temperature=rng.choice([1.0, 1.0, 1.5, 4.0]),
                    dtype=rng.choice(["bf16", "f32"]), labels=k == 0 or rng.random() < 0.7, grad=rng.choice(["none", "with", "with", "later"]))
    M = _log(rng, 1, 64) if rng.random() < 0.4 else _log(rng, 64, 8192)
    return dict(op=op, train=M > 16 and rng.random() < 0.5, M=M, N=8 * _log(rng, 8, 640), K=8 * _log(rng, 8, 400), act=rng.choice(["silu", "gelu"]))


# ------------------------------------------------------------------------------------------------ the format, in 32 bits
def _up(n, m):
    return -(-n // m) * m


def _exponent(top):
    """The e of 2^e for blocks whose largest magnitude is `top`; 448 = 0.875 * 2^9."""
    mant, exp = torch.frexp(top)
    return torch.where(top > 0, exp - 9 + (mant > 0.875), -127).clamp(-127, 127)


def _pow2(e):
    """2^e in fp32 for whole e in [-127, 127], put together from its bits (a power function may be off in the last place)."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _quantize(x):
    """fp32 [rows, cols] -> (codes [rows, cols up to 16], scales)."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, _up(cols, 128) - cols)).view(rows, -1, 128)
    e = _exponent(b.abs().amax(dim=2))
    q = (b * _pow2(-e.unsqueeze(2))).to(F8).view(rows, -1)[:, : _up(cols, 16)].contiguous()
    words = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, _up(e.shape[1], 4) - e.shape[1]))
    return q, words.view(rows, -1, 4).permute(1, 0, 2).contiguous().view(E8)


def _values(q, scales, cols):
    rows = scales.shape[1]
    e = scales.view(torch.uint8).permute(1, 0, 2).reshape(rows, -1).to(torch.int32) - 127
    return q[:, :cols].to(torch.float32) * _pow2(e).repeat_interleave(128, dim=1)[:, :cols]


def _room(rows, cols):
    """Where a result in the block format goes."""
    return (torch.zeros(rows, _up(cols, 16), dtype=torch.uint8, device="cuda").view(F8),
            torch.zeros(_up(_up(cols, 128) // 128, 4) // 4, rows, 4, dtype=torch.uint8, device="cuda").view(E8))


# ------------------------------------------------------------------------------------------------ inputs
def _gauss(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _prepare_scan(case, g, s):
    rows, cols, n, dtype = case["rows"], case["cols"], case["sequences"], TYPES[case["dtype"]]
    # one projection's output holds all three side by side; channels remember from a few to some hundred tokens
    width = 3 if case["gate"] else 2
    s["fvo"] = _gauss(g, rows, width * cols, dtype=dtype)
    bias = torch.rand(cols, generator=g, device="cuda") * 5.0 + 1.0
    s["fvo"][:, :cols] = (s["fvo"][:, :cols].float() + bias).to(dtype)
    s["f"], s["v"] = s["fvo"][:, :cols], s["fvo"][:, cols: 2 * cols]
    s["o"] = s["fvo"][:, 2 * cols:] if case["gate"] else None
    if case["ragged"]:
        last = rows - rows // 50
        cuts = torch.randint(0, last + 1, (n - 1,), generator=g, device="cuda").sort().values
        s["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), last)])
        s["bounds"] = s["offsets"]
    else:
        s["offsets"] = None
        s["bounds"] = torch.arange(n + 1, device="cuda") * (rows // n)
    s["h0"] = _gauss(g, n, cols, scale=0.5) if case["states"] else None
    s["y"] = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    s["h_last"] = torch.zeros(n, cols, device="cuda") if case["states"] else None
    if case["train"]:
        s["dy"] = _gauss(g, rows, cols, scale=1e-2, dtype=dtype)
        s["dh_last"] = _gauss(g, n, cols, scale=1e-2) if case["states"] else None
        s["dh0"] = torch.zeros(n, cols, device="cuda") if case["states"] else None
        s["dfvo"] = torch.zeros(rows, width * cols, dtype=dtype, device="cuda")


def _prepare_loss(case, g, s):
    rows, vocab, k, dtype = case["rows"], case["vocab"], case["k"], TYPES[case["dtype"]]
    # logits as a trained model has them: most words far below the few that fit
    z = _gauss(g, rows, vocab, scale=2.0)
    z[torch.arange(rows, device="cuda").repeat_interleave(4), torch.randint(0, vocab, (4 * rows,), generator=g, device="cuda")] += 8.0
    s["logits"] = z.to(dtype)
    if case["labels"]:
        s["labels"] = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        s["labels"][torch.rand(rows, generator=g, device="cuda") < 0.05] = -100      # padding: no label
    if k:
        # the teacher agrees roughly with the student; some of its lists are shorter than k
        like = z.add_(_gauss(g, rows, vocab))
        top = like.topk(k, dim=1)
        s["teacher_logits"], s["teacher_index"] = top.values.contiguous(), top.indices.to(torch.int32)
        cut = torch.rand(rows, generator=g, device="cuda") < 0.05
        s["teacher_index"][cut, k // 2:] = -1
    s["loss"], s["lse"] = torch.zeros(rows, device="cuda"), torch.zeros(rows, 2, device="cuda")
    if case["grad"] != "none":
        s["dloss"] = torch.rand(rows, generator=g, device="cuda") / rows
        s["dlogits"] = torch.zeros(rows, vocab, dtype=dtype, device="cuda")
    if case["grad"] == "later":      # what the forward pass has left
        d = s["logits"].double()
        s["lse"] = torch.stack([torch.logsumexp(d, 1), torch.logsumexp(d / case["temperature"], 1)], dim=1).float()


def _prepare_ffn(case, g, s):
    M, N, K = case["M"], case["N"], case["K"]
    channel = torch.exp(_gauss(g, K, scale=0.5))
    s["x"], s["x_scale"] = _quantize(_gauss(g, M, K) * channel)
    s["w"], s["w_scale"] = _quantize(_gauss(g, 2 * N, K, scale=1.0 / math.sqrt(K)))
    s["z"], s["z_scale"] = _room(M, N)
    if case["train"]:
        s["gu"] = torch.zeros(M, 2 * N, dtype=BF, device="cuda")
        s["dz"] = (_gauss(g, M, N, scale=1e-3) * torch.exp(_gauss(g, M, 1))).to(BF)
        s["dq"], s["dq_scale"] = _room(M, 2 * N)
        s["dqt"], s["dqt_scale"] = _room(2 * N, M)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    {"scan": _prepare_scan, "loss": _prepare_loss, "ffn": _prepare_ffn}[case["op"]](case, g, s)
    if own:      # argument blocks and workspaces, which a program keeps from step to step
        import paper_2009_02701_b200 as hp
        s["calls"] = _calls(hp, case, s)
    return s


# ------------------------------------------------------------------------------------------------ through the package
def _calls(hp, case, s):
    op, kind = case["op"], {"f32": hp.HPSGD_F32, "bf16": hp.HPSGD_BF16}
    if op == "scan":
        rows, cols, n, dtype = case["rows"], case["cols"], case["sequences"], kind[case["dtype"]]
        ld = s["fvo"].shape[1]
        given = dict(f=s["f"], v=s["v"], o=s["o"], offsets=s["offsets"], h0=s["h0"], ldf=ld, ldv=ld, ldo=ld)
        if case["train"]:
            s["saved"] = torch.empty(hp.hpsgd_gated_scan_saved_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        calls = [(hp.hpsgd_gated_scan_forward, hp.make_gated_scan_forward(rows, cols, n, dtype, y=s["y"], h_last=s["h_last"], saved=s.get("saved"), **given))]
        if case["train"]:
            d = s["dfvo"]
            calls.append((hp.hpsgd_gated_scan_backward,
                          hp.make_gated_scan_backward(rows, cols, n, dtype, saved=s["saved"], dy=s["dy"], df=d[:, :cols], dv=d[:, cols: 2 * cols],
                                                      do=d[:, 2 * cols:] if case["gate"] else None, dh_last=s["dh_last"], dh0=s["dh0"],
                                                      lddf=ld, lddv=ld, lddo=ld, **given)))
        return calls
    if op == "loss":
        a = hp.make_distill_loss(case["rows"], case["vocab"], case["k"], kind[case["dtype"]], logits=s["logits"], labels=s.get("labels"),
                                 teacher_index=s.get("teacher_index"), teacher_logits=s.get("teacher_logits"), temperature=case["temperature"],
                                 label_weight=0.5, teacher_weight=0.5, loss=s["loss"], lse=s["lse"], dlogits=s.get("dlogits"), dloss=s.get("dloss"))
        return [(hp.hpsgd_distill_loss_backward if case["grad"] == "later" else hp.hpsgd_distill_loss, a)]
    M, N, K = case["M"], case["N"], case["K"]
    act = {"silu": hp.HPSGD_SILU, "gelu": hp.HPSGD_GELU}[case["act"]]
    calls = [(hp.hpsgd_gated_ffn_forward, hp.make_gated_ffn_forward(M, N, K, act, s["x"], s["x_scale"], s["w"], s["w_scale"], z8=s["z"], z_scale=s["z_scale"],
                                                                    gu=s.get("gu")))]
    if case["train"]:
        calls.append((hp.hpsgd_gated_ffn_backward, hp.make_gated_ffn_backward(M, N, act, s["gu"], s["dz"], hp.HPSGD_BF16, dq=s["dq"], dq_scale=s["dq_scale"],
                                                                              dqt=s["dqt"], dqt_scale=s["dqt_scale"])))
    return calls


def _outputs(s):
    case = s["case"]
    if case["op"] == "scan":
        names = ["y", "h_last"] + (["dfvo", "dh0"] if case["train"] else [])
    elif case["op"] == "loss":
        names = ["dlogits"] if case["grad"] == "later" else ["loss", "lse", "dlogits"]
    else:
        names = ["z", "z_scale"] + (["gu", "dq", "dq_scale", "dqt", "dqt_scale"] if case["train"] else [])
    return {k: s[k] for k in names if s.get(k) is not None}


def run(s):
    if own:
        for call, args in s["calls"]:
            call(args)
    else:
        {"scan": _run_scan, "loss": _run_loss, "ffn": _run_ffn}[s["case"]["op"]](s)
    return _outputs(s)


# ------------------------------------------------------------------------------------------------ in elementary operations
def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _linear_scan(a, b):
    """h_t = a_t h_(t-1) + b_t down the rows, h before the first being 0, by doubling the distance that is covered."""
    d = 1
    while d < a.shape[0]:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _run_scan(s):
    case, begin, end = s["case"], s["bounds"][:-1], s["bounds"][1:]
    cols, some = case["cols"], s["bounds"][1:] > s["bounds"][:-1]
    first, last = begin[some], end[some] - 1
    f, v = s["f"].float(), s["v"].float()
    a = _sigmoid(f)
    r = 1.0 / (1.0 + torch.exp(f))      # 1 - a, where a is next to 1
    gate = _sigmoid(s["o"].float()) if case["gate"] else 1.0
    keep, x = a.clone(), r * v
    keep[first] = 0.0      # no sequence sees the one before it
    if case["states"]:
        x[first] += a[first] * s["h0"][some]
    inside = torch.arange(case["rows"], device="cuda") < s["bounds"][-1]
    h = _linear_scan(keep, x)
    dtype = s["y"].dtype
    s["y"].copy_(torch.where(inside[:, None], (h * gate).to(dtype), s["y"]))
    if case["states"]:
        s["h_last"].copy_(s["h0"])
        s["h_last"][some] = h[last]
    if not case["train"]:
        return
    dy = s["dy"].float() * inside[:, None]
    g = dy * gate
    if case["states"]:
        g[last] += s["dh_last"][some]
    back = torch.cat([a[1:], a[:1]])
    back[last] = 0.0      # what reaches h_t from h_(t+1)
    G = _linear_scan(back.flip(0), g.flip(0)).flip(0)
    before = torch.cat([h[:1], h[:-1]])
    before[first] = s["h0"][some] if case["states"] else 0.0
    d = [G * (before - v) * a * r, G * r]
    if case["gate"]:
        d.append(dy * h * gate * (1.0 / (1.0 + torch.exp(s["o"].float()))))
    s["dfvo"].copy_((torch.cat(d, dim=1) * inside[:, None]).to(dtype))
    if case["states"]:
        s["dh0"].copy_(s["dh_last"])
        s["dh0"][some] = (a * G)[first]


def _run_loss(s):
    case, rows, T = s["case"], s["case"]["rows"], s["case"]["temperature"]
    z = s["logits"].float()
    at = torch.arange(rows, device="cuda")
    if case["grad"] == "later":
        lse, lse_t = s["lse"][:, 0], s["lse"][:, 1]
    else:
        top = z.amax(dim=1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(dim=1))
        lse_t = lse if T == 1.0 else top / T + torch.log(torch.exp((z - top[:, None]) / T).sum(dim=1))
        s["lse"] = torch.stack([lse, lse_t], dim=1)
    total = torch.zeros(rows, device="cuda")
    if case["labels"]:
        has = s["labels"] >= 0
        label = s["labels"].clamp(min=0)
        total = torch.where(has, 0.5 * (lse - z[at, label]), total)
    if case["k"]:
        there = s["teacher_index"] >= 0
        index = s["teacher_index"].clamp(min=0).long()
        t = torch.where(there, s["teacher_logits"] / T, -math.inf)
        e = torch.exp(t - t.amax(dim=1, keepdim=True))
        p = e / e.sum(dim=1, keepdim=True)
        logp = t - t.amax(dim=1, keepdim=True) - torch.log(e.sum(dim=1, keepdim=True))
        logq = z.gather(1, index) / T - lse_t[:, None]
        total = total + 0.5 * T * T * torch.where(there, p * (logp - logq), 0.0).sum(dim=1)
    s["loss"] = total
    if case["grad"] == "none":
        return
    d = torch.zeros_like(z)
    if case["labels"]:
        d += torch.exp(z - lse[:, None]) * (0.5 * has)[:, None]
        d[at, label] -= 0.5 * has
    if case["k"]:
        d += torch.exp(z / T - lse_t[:, None]) * (0.5 * T)
        d.scatter_add_(1, index, p * (-0.5 * T))
    s["dlogits"] = (d * s["dloss"][:, None]).to(s["logits"].dtype)


def _act(x, kind):
    """act(x) and its derivative."""
    if kind == "silu":
        p = _sigmoid(x)
        return x * p, p * (1.0 + x * (1.0 - p))
    t = torch.tanh(GELU_1 * (x + GELU_3 * x * x * x))
    return 0.5 * x * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * GELU_1 * (1.0 + 3.0 * GELU_3 * x * x)


def _run_ffn(s):
    case, N, K = s["case"], s["case"]["N"], s["case"]["K"]
    y = _values(s["x"], s["x_scale"], K) @ _values(s["w"], s["w_scale"], K).t()
    s["z"], s["z_scale"] = _quantize(_act(y[:, :N], case["act"])[0] * y[:, N:])
    if case["train"]:
        s["gu"] = y.to(BF)
        g, u, dz = s["gu"][:, :N].float(), s["gu"][:, N:].float(), s["dz"].float()
        a, da = _act(g, case["act"])
        d = torch.cat([dz * u * da, dz * a], dim=1)
        s["dq"], s["dq_scale"] = _quantize(d)
        s["dqt"], s["dqt_scale"] = _quantize(d.t().contiguous())


# ------------------------------------------------------------------------------------------------ cost
def work(case):
    op, size = case["op"], {"f32": 4, "bf16": 2}
    if op == "scan":
        n, t = case["rows"] * case["cols"], size[case["dtype"]]
        wide = 3 if case["gate"] else 2
        state = 4 * case["sequences"] * case["cols"] if case["states"] else 0
        if case["train"]:
            return {"bytes": n * t * (wide + 1 + wide + 1 + wide) + 4 * state, "flops": 30 * n}
        return {"bytes": n * t * (wide + 1) + 2 * state, "flops": 12 * n}
    if op == "loss":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size[case["dtype"]] * (1 if case["grad"] == "none" else 2) + case["rows"] * (8 * case["k"] + 24), "flops": 8 * n}
    M, N, K = case["M"], case["N"], case["K"]
    bytes_ = (M + 2 * N) * K * (1 + 1 / 128) + M * N * (1 + 1 / 128)
    return {"bytes": bytes_ + (M * N * (4 + 4 + 2 + 4) if case["train"] else 0), "flops": 4 * M * N * K + (30 * M * N if case["train"] else 0)}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _two(e):
    """2.0 ** e in 64 bits for whole e, exactly."""
    return torch.bitwise_left_shift(e.to(torch.int64) + 1023, 52).view(torch.float64)


def _q64(x):
    """64-bit [rows, cols] -> values of the codes and of the scales in their array."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    b = torch.zeros(rows, nb * 128, dtype=torch.float64, device=x.device)
    b[:, :cols] = x
    b = b.view(rows, nb, 128)
    top = b.abs().amax(dim=2)
    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448.0))      # and one correction each way
    e = torch.where(448.0 * _two(e - 1) >= top, e - 1, e)
    e = torch.where(448.0 * _two(e) < top, e + 1, e).clamp(-127.0, 127.0)
    w = b / _two(e.unsqueeze(2))
    step = _two(torch.frexp(torch.clamp(w.abs(), min=2.0 ** -6))[1] - 4)
    q = torch.round(w / step) * step      # (round: halves to even)
    full = torch.full((rows, -(-nb // 4) * 4), -127.0, dtype=torch.float64, device=x.device)
    full[:, :nb] = e
    return q.view(rows, -1)[:, : -(-cols // 16) * 16], _two(full.view(rows, -1, 4).transpose(0, 1))


def _v64(q, scale, cols):
    f = scale.to(torch.float32).double().transpose(0, 1).reshape(q.shape[0], -1)
    at = torch.arange(cols, device=q.device) // 128
    return q[:, :cols].to(torch.float32).double() * f[:, at]


def _exact_scan(case, s):
    """Step by step through time, all sequences at once, the longest first."""
    bounds = s["bounds"].cpu()
    length = bounds[1:] - bounds[:-1]
    order = torch.argsort(length, descending=True, stable=True)
    sorted_length, begin = length[order], bounds[:-1][order].cuda()
    longest, rows, cols, n = int(length.max()), case["rows"], case["cols"], case["sequences"]
    active = [int(x) for x in torch.searchsorted(-sorted_length, -torch.arange(longest), right=False)]      # sequences longer than t
    place = order.cuda()
    f, v = s["f"].double(), s["v"].double()
    a = torch.sigmoid(f)
    r = torch.sigmoid(-f)
    zero = torch.zeros(n, cols, dtype=torch.float64, device="cuda")
    h0 = s["h0"].double()[place] if case["states"] else zero
    h, state, before = torch.zeros(rows, cols, dtype=torch.float64, device="cuda"), h0.clone(), torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    inflow = r * v
    for t in range(longest):
        k = active[t]
        at = begin[:k] + t
        before[at] = state[:k]
        state[:k] = torch.addcmul(inflow[at], a[at], state[:k])
        h[at] = state[:k]
    inside = (torch.arange(rows, device="cuda") < int(bounds[-1]))[:, None]
    gate = torch.sigmoid(s["o"].double()) if case["gate"] else torch.ones_like(h)
    out = {"y": h * gate * inside}
    if case["states"]:
        out["h_last"] = torch.empty_like(zero)
        out["h_last"][place] = state
    if not case["train"]:
        return out
    dy = s["dy"].double() * inside
    g = dy * gate
    flow = s["dh_last"].double()[place] if case["states"] else zero.clone()      # the gradient that reaches h_t from behind
    G = torch.zeros_like(h)
    for t in reversed(range(longest)):
        k = active[t]
        at = begin[:k] + t
        now = g[at] + flow[:k]
        G[at] = now
        flow[:k] = now * a[at]
    parts = [G * (before - v) * a * r, G * r] + ([dy * h * gate * torch.sigmoid(-s["o"].double())] if case["gate"] else [])
    out["dfvo"] = torch.cat(parts, dim=1)
    if case["states"]:
        out["dh0"] = torch.empty_like(zero)
        out["dh0"][place] = flow
    return out


def _exact_loss(case, s):
    T, rows, out = case["temperature"], case["rows"], {"loss": [], "lse": [], "dlogits": []}
    step = max(1, 2 ** 26 // case["vocab"])
    for i in range(0, rows, step):      # a few rows at a time: 64 bits of a whole batch are many
        z = s["logits"][i: i + step].double()
        lse = torch.stack([torch.logsumexp(z, 1), torch.logsumexp(z / T, 1)], dim=1)
        if case["grad"] == "later":
            lse = s["lse"][i: i + step].double()
        total = torch.zeros(len(z), dtype=torch.float64, device="cuda")
        d = torch.zeros_like(z)
        at = torch.arange(len(z), device="cuda")
        if case["labels"]:
            label = s["labels"][i: i + step]
            rows_with, of = at[label >= 0], label[label >= 0]
            total[rows_with] += 0.5 * (lse[rows_with, 0] - z[rows_with, of])
            d[rows_with] += 0.5 * torch.exp(z[rows_with] - lse[rows_with, :1])
            d[rows_with, of] -= 0.5
        if case["k"]:
            index, t = s["teacher_index"][i: i + step].long(), s["teacher_logits"][i: i + step].double() / T
            t = t.masked_fill(index < 0, -math.inf)
            p = torch.softmax(t, dim=1)
            at_k = index.clamp(min=0)
            term = torch.xlogy(p, p) - p * (torch.gather(z, 1, at_k) / T - lse[:, 1:])
            total += 0.5 * T ** 2 * term.sum(dim=1)
            d += 0.5 * T * torch.exp(z / T - lse[:, 1:])
            d.scatter_add_(1, at_k, -0.5 * T * p)
        out["loss"].append(total)
        out["lse"].append(lse)
        if case["grad"] != "none":
            out["dlogits"].append(d * s["dloss"][i: i + step].double()[:, None])
    names = {"none": ("loss", "lse"), "with": ("loss", "lse", "dlogits"), "later": ("dlogits",)}[case["grad"]]
    return {k: torch.cat(out[k]) for k in names}


def _act64(x, kind):
    if kind == "silu":
        return x * torch.sigmoid(x), torch.sigmoid(x) + x * torch.sigmoid(x) * torch.sigmoid(-x)
    w = 2.0 * GELU_1 * (x + GELU_3 * x ** 3)      # (1 + tanh(w / 2)) / 2 = sigmoid(w)
    return x * torch.sigmoid(w), torch.sigmoid(w) + x * torch.sigmoid(w) * torch.sigmoid(-w) * 2.0 * GELU_1 * (1.0 + 3.0 * GELU_3 * x ** 2)


def _exact_ffn(case, s):
    N, K = case["N"], case["K"]
    x, w = _v64(s["x"], s["x_scale"], K), _v64(s["w"], s["w_scale"], K)
    g, u = x @ w[:N].t(), x @ w[N:].t()
    out = {}
    out["z"], out["z_scale"] = _q64(_act64(g, case["act"])[0] * u)
    if case["train"]:
        out["gu"] = torch.cat([g, u], dim=1)
        g, u = g.to(BF).double(), u.to(BF).double()      # they are kept, and taken up again, in bf16
        a, da = _act64(g, case["act"])
        dz = s["dz"].double()
        d = torch.cat([dz * u * da, dz * a], dim=1)
        out["dq"], out["dq_scale"] = _q64(d)
        out["dqt"], out["dqt_scale"] = _q64(d.t().contiguous())
    return out


def exact(case, seed):
    s = prepare(dict(case), seed)
    return {"scan": _exact_scan, "loss": _exact_loss, "ffn": _exact_ffn}[case["op"]](case, s)
