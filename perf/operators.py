"""Cases for measuring the low-precision training operators: the AdamW step over many tensors (with the global
norm that clips its gradients), the root-mean-square norm with the residual's addition and an 8-bit output, the
8-bit block format itself, and the matrix product on that format.

``run`` computes them in elementary torch operations where ``own`` is false, and through the package's entry
points where it is true.  ``exact`` restates their definitions in 64 bits.

The 8-bit block format: a matrix [rows, cols] is held as E4M3 codes and one power of two (E8M0) for every 128
consecutive columns of a row, the smallest 2^e >= 2^-127 with 448 * 2^e >= the block's largest magnitude.  Codes
are [rows, cols up to a multiple of 16]; the scale of block b of row r is entry [b // 4, r, b % 4] of an array
[ceil(blocks / 4), rows, 4].
"""
import math
import random

import torch

own = False

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, BETA1, BETA2, EPS, DECAY, STEP, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1000, 1.0
NORM_EPS = 1e-5
M1, M2, M3 = 0x6A09E667, 0xBB67AE85, 0x3C6EF373      # frac(sqrt 2, 3, 5) * 2^32 with the low bit set


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # a few small tensors: the whole step is a launch (biases and norms of one layer, one ragged matrix)
        dict(name="adamw32 3 tensors", op="adamw", tensors=3, total=204_176, bits=32, grad="f32", param="f32", copy=False, clip=False),
        # a model of 62 tensors: gradients from bf16 layers, fp32 weights with the bf16 copy that the next forward reads
        dict(name="adamw32 62 tensors clip", op="adamw", tensors=62, total=11_700_000, bits=32, grad="bf16", param="f32", copy=True, clip=True),
        # the fully connected layout: 138 M weights, all in 32 bits
        dict(name="adamw32 138M clip", op="adamw", tensors=32, total=138_000_000, bits=32, grad="f32", param="f32", copy=False, clip=True),
        # 161 tensors with both moments in 8 bits
        dict(name="adamw8 161 tensors clip", op="adamw", tensors=161, total=25_600_000, bits=8, grad="f32", param="f32", copy=False, clip=True),
        # the fully connected layout at its smallest: bf16 weights and gradients, moments in 8 bits
        dict(name="adamw8 138M bf16", op="adamw", tensors=32, total=138_000_000, bits=8, grad="bf16", param="bf16", copy=False, clip=False),
        # the norm in front of a layer while one token is generated
        dict(name="norm 1 token", op="norm_forward", rows=1, cols=1024, dtype="bf16", residual=True),
        # the same over a batch of sequences
        dict(name="norm 16384 tokens", op="norm_forward", rows=16384, cols=4096, dtype="bf16", residual=True),
        # its backward pass, with a row count and a width that no tile divides
        dict(name="norm backward ragged", op="norm_backward", rows=8191, cols=2008, dtype="bf16", residual=True),
        # one token against an output projection of 30000 words
        dict(name="product 1 token", op="product", M=1, N=30000, K=1024, out="f32"),
        # a layer's forward over a batch of sequences
        dict(name="product 8192 tokens", op="product", M=8192, N=4096, K=4096, out="bf16"),
        # a layer's backward: the gradient quantised both ways, the input's gradient, the weight's added to what is there
        dict(name="linear backward ragged", op="linear_backward", M=4095, N=4096, K=1024),
        # the embedding or the projection after an optimizer step, laid out for the forward and for the backward
        dict(name="quantize 30000 x 1024", op="quantize", rows=30000, cols=1024, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "norm_forward", "norm_backward", "product", "product", "linear_backward", "quantize"])
    if op == "adamw":
        tensors = _log(rng, 1, 600)
        bits = rng.choice([8, 32])
        param = rng.choice(["f32", "f32", "bf16"])
        return dict(op=op, tensors=tensors, total=max(tensors, _log(rng, 1000, 100_000_000)), bits=bits,
                    grad=rng.choice(["f32", "bf16"]), param=param, copy=param == "f32" and rng.random() < 0.5, clip=rng.random() < 0.5)
    if op in ("norm_forward", "norm_backward"):
        cols = _log(rng, 32, 8192)
        if rng.random() < 0.7:
            cols = -(-cols // 8) * 8
        rows = _log(rng, 1 if op == "norm_forward" else 16, 16384)
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7)
    if op == "quantize":
        return dict(op=op, rows=_log(rng, 16, 16384), cols=_log(rng, 64, 8192), dtype=rng.choice(["bf16", "f32"]))
    if op == "product":
        M = _log(rng, 1, 64) if rng.random() < 0.5 else _log(rng, 64, 8192)
        return dict(op=op, M=M, N=_log(rng, 128, 8192), K=_log(rng, 64, 4096), out=rng.choice(["bf16", "f32"]))
    return dict(op=op, M=_log(rng, 64, 8192), N=8 * _log(rng, 16, 512), K=8 * _log(rng, 16, 512))


# ------------------------------------------------------------------------------------------------ the format, in 32 bits
def _up(n, m):
    return -(-n // m) * m


def _blocks(x):
    """[rows, cols] in 32 bits -> [rows, blocks, 128], zeros behind the last column."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, _up(cols, 128) - cols)).view(rows, -1, 128)


def _exponent(top):
    """The e of 2^e for blocks whose largest magnitude is `top`; 448 = 0.875 * 2^9."""
    mant, exp = torch.frexp(top)
    return torch.where(top > 0, exp - 9 + (mant > 0.875), -127).clamp(-127, 127)


def _pow2(e):
    """2^e in fp32 for whole e in [-127, 127], put together from its bits (a power function may be off in the last place)."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _scale_array(e):
    """Exponents [rows, blocks] -> E8M0 [ceil(blocks / 4), rows, 4]."""
    rows, blocks = e.shape
    words = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, _up(blocks, 4) - blocks))
    return words.view(rows, -1, 4).permute(1, 0, 2).contiguous().view(E8)


def _scale_of(scales, cols):
    """E8M0 [ceil(blocks / 4), rows, 4] -> fp32 factors [rows, cols]."""
    rows = scales.shape[1]
    e = scales.view(torch.uint8).permute(1, 0, 2).reshape(rows, -1).to(torch.int32) - 127
    return _pow2(e).repeat_interleave(128, dim=1)[:, :cols]


def _quantize(x):
    """fp32 [rows, cols] -> (codes [rows, cols up to 16], scales)."""
    rows, cols = x.shape
    b = _blocks(x)
    e = _exponent(b.abs().amax(dim=2))
    q = (b * _pow2(-e.unsqueeze(2))).to(F8).view(rows, -1)[:, : _up(cols, 16)].contiguous()
    return q, _scale_array(e)


def _values(q, scales, cols):
    return q[:, :cols].to(torch.float32) * _scale_of(scales, cols)


# ------------------------------------------------------------------------------------------------ inputs
def _sizes(case, seed):
    """Tensor sizes, log-uniform over four decades, that add up to the case's total."""
    r = random.Random(1000 + case["tensors"])
    raw = [math.exp(r.uniform(0.0, math.log(10_000.0))) for _ in range(case["tensors"])]
    k = case["total"] / sum(raw)
    sizes = [max(1, int(k * x)) for x in raw]
    sizes[sizes.index(max(sizes))] += max(0, case["total"] - sum(sizes))
    return sizes


def _gauss(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _activations(g, rows, cols, dtype):
    """Normal values with a few channels that are much larger, as the residual stream of a trained model has them."""
    channel = torch.exp(_gauss(g, cols, scale=0.5))
    channel[torch.randint(0, cols, (max(1, cols // 256),), generator=g, device="cuda")] *= 20.0
    return (_gauss(g, rows, cols) * channel).to(dtype)


def _gradients(g, n):
    """Normal values of widely spread sizes; one run of 64 in ten has none (rows that no token of the batch used)."""
    x = _gauss(g, n, scale=1e-3)
    k = _up(n, 64) // 64
    size = torch.exp(_gauss(g, k)) * (torch.rand(k, generator=g, device="cuda") >= 0.1)
    return x.mul_(size.repeat_interleave(64)[:n])


def _prepare_adamw(case, g, seed):
    sizes = _sizes(case, seed)
    starts, pos = [], 0
    for n in sizes:
        starts.append(pos)
        pos += _up(n, 128)
    s = {"n": pos, "sizes": sizes, "starts": starts, "seed": seed & 0x7FFFFFFF}
    live = torch.zeros(pos + 1, dtype=torch.int8, device="cuda")
    at = torch.tensor(starts, device="cuda")
    live[at] += 1
    live[at + torch.tensor(sizes, device="cuda")] -= 1
    live = live[:pos].cumsum(0, dtype=torch.int8)
    s["param"] = (_gauss(g, pos, scale=0.05) * live).to(TYPES[case["param"]])
    grad = _gradients(g, pos) * live
    s["grad"] = grad.to(TYPES[case["grad"]])
    m = _gradients(g, pos).mul_(0.3) * live
    v = (_gauss(g, pos, scale=0.7) * grad).square_().add_(1e-8) * live
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        for name, x in (("m", m), ("r", v.sqrt())):
            q, sc = _quantize(x.view(1, -1))
            s[name] = q.view(-1)
            s[name + "_scale"] = sc.view(torch.uint8).view(-1)[: pos // 128].clone().view(E8)
    if case["copy"]:
        s["copy"] = torch.zeros(pos, dtype=torch.bfloat16, device="cuda")
    s["norm"] = torch.zeros(2, device="cuda")
    if own:      # the table of tensors and the norm's workspace, which a training program builds once
        import paper_2009_02701_b200 as hp
        names = ("m", "v") if case["bits"] == 32 else ("m", "r")
        kind = {"f32": hp.HPSGD_F32, "bf16": hp.HPSGD_BF16}
        rows = []
        for start, n in zip(starts, sizes):
            row = {"param": s["param"][start:], "grad": s["grad"][start:], "m": s[names[0]][start:], "v": s[names[1]][start:],
                   "n": n, "weight_decay": DECAY, "rng_offset": start}
            if case["bits"] == 8:
                row |= {"m_scale": s["m_scale"][start // 128:], "v_scale": s["r_scale"][start // 128:]}
            if case["copy"]:
                row["copy"] = s["copy"][start:]
            rows.append(row)
        s["table"] = hp.make_adamw_table(rows, kind[case["param"]], kind[case["grad"]], case["bits"])
        s["workspace"] = torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    if op == "adamw":
        return {"case": case, **_prepare_adamw(case, g, seed)}
    s = {"case": case}
    new = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731

    def room(rows, cols):      # where an 8-bit result goes
        return (torch.zeros(rows, _up(cols, 16), dtype=torch.uint8, device="cuda").view(F8),
                torch.zeros(_up(_up(cols, 128) // 128, 4) // 4, rows, 4, dtype=torch.uint8, device="cuda").view(E8))

    if op in ("norm_forward", "norm_backward"):
        rows, cols, dtype = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"] = _activations(g, rows, cols, dtype)
        s["weight"] = (1.0 + _gauss(g, cols, scale=0.1)).to(dtype)
        if op == "norm_forward":
            if case["residual"]:
                s["residual"] = _activations(g, rows, cols, dtype)
                s["h"] = new(rows, cols, dtype=dtype)
            s["y"], s["y_scale"] = room(rows, cols)
            s["rstd"] = new(rows, dtype=torch.float32)
        else:
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(dim=1) + NORM_EPS)
            s["dy"] = _gauss(g, rows, cols, scale=1e-3, dtype=dtype)
            if case["residual"]:
                s["dres"] = _gauss(g, rows, cols, scale=1e-3, dtype=dtype)
            s["dx"], s["dweight"] = new(rows, cols, dtype=dtype), new(cols, dtype=torch.float32)
    elif op == "quantize":
        s["x"] = _gauss(g, case["rows"], case["cols"], scale=0.02).mul_(torch.exp(_gauss(g, case["rows"], 1))).to(TYPES[case["dtype"]])
        s["q"], s["scale"] = room(case["rows"], case["cols"])
        s["qt"], s["scale_t"] = room(case["cols"], case["rows"])
    else:
        M, N, K = case["M"], case["N"], case["K"]
        s["x"], s["x_scale"] = _quantize(_activations(g, M, K, torch.float32))
        w = _gauss(g, N, K, scale=0.02)
        if op == "product":
            s["w"], s["w_scale"] = _quantize(w)
            s["y"] = new(M, N, dtype=TYPES[case["out"]])
        else:
            s["wt"], s["wt_scale"] = _quantize(w.t().contiguous())
            s["dy"] = (_gauss(g, M, N, scale=1e-3) * torch.exp(_gauss(g, M, 1))).to(torch.bfloat16)
            s["dyq"], s["dyq_scale"] = room(M, N)
            s["dyt"], s["dyt_scale"] = room(N, M)
            s["xt"], s["xt_scale"] = room(K, M)
            s["dx"] = new(M, K, dtype=torch.bfloat16)
            s["dw"] = _gauss(g, N, K, scale=1e-2)
    if own:      # argument blocks and workspaces, which a program keeps from step to step
        import paper_2009_02701_b200 as hp
        s["calls"] = _calls(hp, case, s)
    return s


# ------------------------------------------------------------------------------------------------ through the package
def _calls(hp, case, s):
    op, kind = case["op"], {"f32": hp.HPSGD_F32, "bf16": hp.HPSGD_BF16}
    if op == "norm_forward":
        a = hp.make_rmsnorm_forward(case["rows"], case["cols"], NORM_EPS, kind[case["dtype"]], x=s["x"], residual=s.get("residual"),
                                    weight=s["weight"], h=s.get("h"), y8=s["y"], y_scale=s["y_scale"], rstd=s["rstd"])
        return [(hp.hpsgd_rmsnorm_forward, a)]
    if op == "norm_backward":
        s["workspace"] = torch.zeros(hp.hpsgd_rmsnorm_backward_bytes(case["rows"], case["cols"]), dtype=torch.uint8, device="cuda")
        a = hp.make_rmsnorm_backward(case["rows"], case["cols"], kind[case["dtype"]], h=s["x"], weight=s["weight"], rstd=s["rstd"], dy=s["dy"],
                                     dres=s.get("dres"), dx=s["dx"], dweight=s["dweight"], workspace=s["workspace"])
        return [(hp.hpsgd_rmsnorm_backward, a)]
    if op == "quantize":
        return [(hp.hpsgd_quantize_fp8, hp.make_quantize_fp8(case["rows"], case["cols"], kind[case["dtype"]], s["x"], q=s["q"],
                                                             scale=s["scale"], qt=s["qt"], scale_t=s["scale_t"]))]
    M, N, K = case["M"], case["N"], case["K"]
    s["workspace"] = []

    def product(m, n, k, a, sa, b, sb, d, dtype, accumulate=False):
        s["workspace"].append(torch.zeros(hp.hpsgd_gemm_fp8_bytes(m, n, k), dtype=torch.uint8, device="cuda"))
        return (hp.hpsgd_gemm_fp8, hp.make_gemm_fp8(m, n, k, a, sa, b, sb, d, dtype, accumulate=accumulate, workspace=s["workspace"][-1]))

    if op == "product":
        return [product(M, N, K, s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"], kind[case["out"]])]
    return [(hp.hpsgd_quantize_fp8, hp.make_quantize_fp8(M, N, hp.HPSGD_BF16, s["dy"], q=s["dyq"], scale=s["dyq_scale"], qt=s["dyt"], scale_t=s["dyt_scale"])),
            (hp.hpsgd_quantize_fp8, hp.make_quantize_fp8(M, K, hp.HPSGD_FP8, s["x"], x_scale=s["x_scale"], qt=s["xt"], scale_t=s["xt_scale"])),
            product(M, K, N, s["dyq"], s["dyq_scale"], s["wt"], s["wt_scale"], s["dx"], hp.HPSGD_BF16),
            product(N, K, M, s["dyt"], s["dyt_scale"], s["xt"], s["xt_scale"], s["dw"], hp.HPSGD_F32, accumulate=True)]


def _run_own(s):
    case = s["case"]
    if case["op"] == "adamw":
        import paper_2009_02701_b200 as hp
        scale = None
        if case["clip"]:
            hp.hpsgd_grad_norm(s["table"], MAX_NORM, s["workspace"], s["norm"])
            scale = s["norm"][1:]
        hp.hpsgd_adamw_step(s["table"], LR, BETA1, BETA2, EPS, STEP, s["seed"], scale)
    else:
        for call, args in s["calls"]:
            call(args)
    return _outputs(s)


def _outputs(s):
    names = {"adamw": ("param", "m", "v", "r", "m_scale", "r_scale", "copy"), "norm_forward": ("h", "y", "y_scale", "rstd"),
             "norm_backward": ("dx", "dweight"), "product": ("y",), "quantize": ("q", "scale", "qt", "scale_t"),
             "linear_backward": ("dyq", "dyq_scale", "dyt", "dyt_scale", "xt", "xt_scale", "dx", "dw")}[s["case"]["op"]]
    out = {k: s[k] for k in names if k in s}
    if s["case"].get("clip"):
        out["norm"] = s["norm"]
    return out


# ------------------------------------------------------------------------------------------------ in elementary operations
def _key(seed, step):
    """The two 32-bit keys of a step's random bits: the counter hash of this repository's gradients over (seed, step)."""
    mask = (1 << 64) - 1
    c = (0x6A09E667F3BCC909, 0xBB67AE8584CAA73B, 0x3C6EF372FE94F82B, 0xA54FF53A5F1D36F1)

    def mix(x):
        x ^= x >> 32
        x = x * c[0] & mask
        x ^= x >> 29
        x = x * c[1] & mask
        return x ^ (x >> 32)

    k = mix((mix((seed + c[2]) & mask) ^ step) + c[3] & mask)
    return k & 0xFFFFFFFF, k >> 32


def _bits(seed, step, n):
    """32 random bits for each of n elements (positions below 2^32), as int64."""
    k0, k1 = _key(seed, step)
    low = 0xFFFFFFFF
    x = torch.arange(n, dtype=torch.int64, device="cuda").bitwise_xor_(k0).mul_(M1).bitwise_and_(low)
    x ^= x >> 15
    x.add_(k1).mul_(M2).bitwise_and_(low)
    x ^= x >> 14
    x.mul_(M3).bitwise_and_(low)
    x ^= x >> 16
    return x


def _float_of(code):
    """E4M3 codes without sign, as integers -> fp32: their bits are the top of a binary32 that is 2^120 times smaller."""
    return (code << 20).view(torch.float32) * 2.0 ** 120


def _step8(m, v, rnd):
    """New moments in 32 bits -> codes and scales.  The first moment is rounded so that its expected value is kept, the second as
    a square root, so that the expected square is; a positive second moment never becomes 0."""
    b = m.view(-1, 128)
    em = _exponent(b.abs().amax(dim=1))
    x = (b * _pow2(-em.unsqueeze(1))).view(-1)
    lo = (x.abs() * 2.0 ** -120).view(torch.int32)
    code = (lo + ((rnd >> 16).to(torch.int32) * 16 + 8)) >> 20
    m8 = (code + torch.where(x < 0, 128, 0)).to(torch.uint8).view(F8)
    r = v.sqrt()
    er = _exponent(r.view(-1, 128).amax(dim=1))
    x = (r.view(-1, 128) * _pow2(-er.unsqueeze(1))).view(-1)
    code = (x * 2.0 ** -120).view(torch.int32) >> 20
    a, b = _float_of(code), _float_of(code + 1)
    u = ((rnd & 0xFFFF).to(torch.float32) + 0.5) * 2.0 ** -16
    code = code + (u * ((b - a) * (b + a)) < (x - a) * (x + a))
    code = torch.where(r > 0, code.clamp(min=1), code)
    return m8, (em + 127).to(torch.uint8).view(E8), code.to(torch.uint8).view(F8), (er + 127).to(torch.uint8).view(E8)


def _factor(scale):
    e = scale.view(torch.uint8).to(torch.int32) - 127
    return _pow2(e).repeat_interleave(128)


def _run_adamw(s):
    case, n = s["case"], s["n"]
    g = s["grad"].float()
    if case["clip"]:
        norm = g.square().sum().sqrt()
        s["norm"] = torch.stack([norm, torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))])
        g = g * s["norm"][1]
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = s["m"].float() * _factor(s["m_scale"])
        v = (s["r"].float() * _factor(s["r_scale"])).square()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    p = s["param"].float() * (1 - LR * DECAY)
    p = p - (LR / (1 - BETA1 ** STEP)) * (m / (v.sqrt() * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS))
    rnd = _bits(s["seed"], STEP, n) if case["bits"] == 8 or case["param"] == "bf16" else None
    if case["param"] == "bf16":      # rounded so that the expected value is kept: steps far below its 8 bits still count
        rnd16 = (rnd * M2 & 0xFFFFFFFF) >> 16
        p = ((p.view(torch.int32) + rnd16.to(torch.int32)) & -65536).view(torch.float32)
    s["param"].copy_(p)
    if case["copy"]:
        s["copy"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for k, x in zip(("m", "m_scale", "r", "r_scale"), _step8(m, v, rnd)):
            s[k].view(torch.uint8).copy_(x.view(torch.uint8))
    return _outputs(s)


def run(s):
    if own:
        return _run_own(s)
    case, op = s["case"], s["case"]["op"]
    if op == "adamw":
        return _run_adamw(s)
    if op == "norm_forward":
        h = s["x"]
        if case["residual"]:
            h = (h.float() + s["residual"].float()).to(h.dtype)
            s["h"] = h
        f = h.float()
        s["rstd"] = torch.rsqrt(f.square().mean(dim=1) + NORM_EPS)
        s["y"], s["y_scale"] = _quantize(f * s["rstd"].unsqueeze(1) * s["weight"].float())
    elif op == "norm_backward":
        x = s["x"].float() * s["rstd"].unsqueeze(1)
        dy = s["dy"].float()
        d = dy * s["weight"].float()
        dx = (d - x * (d * x).mean(dim=1, keepdim=True)) * s["rstd"].unsqueeze(1)
        s["dx"] = (dx + s["dres"].float() if case["residual"] else dx).to(s["x"].dtype)
        s["dweight"] = (dy * x).sum(dim=0)
    elif op == "quantize":
        x = s["x"].float()
        s["q"], s["scale"] = _quantize(x)
        s["qt"], s["scale_t"] = _quantize(x.t().contiguous())
    elif op == "product":
        K = case["K"]
        s["y"] = (_values(s["x"], s["x_scale"], K) @ _values(s["w"], s["w_scale"], K).t()).to(TYPES[case["out"]])
    else:
        M, N, K = case["M"], case["N"], case["K"]
        dy = s["dy"].float()
        s["dyq"], s["dyq_scale"] = _quantize(dy)
        s["dyt"], s["dyt_scale"] = _quantize(dy.t().contiguous())
        s["xt"], s["xt_scale"] = _quantize(_values(s["x"], s["x_scale"], K).t().contiguous())
        s["dx"] = (_values(s["dyq"], s["dyq_scale"], N) @ _values(s["wt"], s["wt_scale"], N).t()).to(torch.bfloat16)
        s["dw"] = s["dw"] + _values(s["dyt"], s["dyt_scale"], M) @ _values(s["xt"], s["xt_scale"], M).t()
    return _outputs(s)


# ------------------------------------------------------------------------------------------------ cost
def work(case):
    op, size = case["op"], {"f32": 4, "bf16": 2}
    if op == "adamw":
        n = case["total"]
        state = 8 if case["bits"] == 32 else 2 + 2 / 128
        per = 2 * size[case["param"]] + size[case["grad"]] * (2 if case["clip"] else 1) + 2 * state + (2 if case["copy"] else 0)
        return {"bytes": n * per, "flops": 14 * n}      # with clipping the gradients have to be known whole before the first is used
    if op in ("norm_forward", "norm_backward"):
        n, t = case["rows"] * case["cols"], size[case["dtype"]]
        if op == "norm_forward":
            return {"bytes": n * (t * (3 if case["residual"] else 1) + 1 + 1 / 128) + case["cols"] * t + 4 * case["rows"], "flops": 6 * n}
        return {"bytes": n * t * (4 if case["residual"] else 3) + case["cols"] * (t + 4) + 4 * case["rows"], "flops": 10 * n}
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + 2 + 2 / 128), "flops": 4 * n}
    M, N, K = case["M"], case["N"], case["K"]
    if op == "product":
        return {"bytes": (M + N) * K * (1 + 1 / 128) + M * N * size[case["out"]], "flops": 2 * M * N * K}
    return {"bytes": M * N * (2 + 2) + M * K * (1 + 1 + 2) + N * K * (1 + 8), "flops": 4 * M * N * K}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _two(e):
    """2.0 ** e in 64 bits for whole e, exactly."""
    return torch.bitwise_left_shift(e.to(torch.int64) + 1023, 52).view(torch.float64)


def _e64(top):
    """Smallest e >= -127 with 448 * 2^e >= top, by its logarithm and one correction each way."""
    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448.0))
    e = torch.where(448.0 * _two(e - 1) >= top, e - 1, e)
    e = torch.where(448.0 * _two(e) < top, e + 1, e)
    return e.clamp(-127.0, 127.0)


def _grid64(x):
    """For x in [0, 448]: the largest E4M3 value <= x, and the distance to the next one."""
    step = _two(torch.frexp(torch.clamp(x, min=2.0 ** -6))[1] - 4)
    return torch.floor(x / step) * step, step


def _nearest64(x):
    lo, step = _grid64(x.abs())
    up = x.abs() - lo
    odd = torch.remainder(torch.round(lo / step), 2.0) == 1.0
    return torch.sign(x) * (lo + step * ((up > step / 2) | ((up == step / 2) & odd)))


def _q64(x, cols16=True):
    """64-bit [rows, cols] -> values of the codes, of the scales in their array, and of their products."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    b = torch.zeros(rows, nb * 128, dtype=torch.float64, device=x.device)
    b[:, :cols] = x
    b = b.view(rows, nb, 128)
    e = _e64(b.abs().amax(dim=2))
    q = _nearest64(b / _two(e.unsqueeze(2)))
    full = torch.full((rows, -(-nb // 4) * 4), -127.0, dtype=torch.float64, device=x.device)
    full[:, :nb] = e
    scale = _two(full.view(rows, -1, 4).transpose(0, 1))
    return q.view(rows, -1)[:, : -(-cols // 16) * 16], scale, (q * _two(e.unsqueeze(2))).view(rows, -1)[:, :cols]


def _v64(q, scale, cols):
    f = scale.to(torch.float32).double().transpose(0, 1).reshape(q.shape[0], -1)
    at = torch.arange(cols, device=q.device) // 128
    return q[:, :cols].to(torch.float32).double() * f[:, at]


def _exact_adamw(case, s):
    g = s["grad"].double()
    out = {}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = torch.stack([norm, torch.clamp(MAX_NORM / norm, max=1.0)])
        g = g * out["norm"][1]
    n = s["n"]
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        at = torch.arange(n, device="cuda") // 128
        m = s["m"].to(torch.float32).double() * s["m_scale"].to(torch.float32).double()[at]
        v = (s["r"].to(torch.float32).double() * s["r_scale"].to(torch.float32).double()[at]) ** 2
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    hat = (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
    p = s["param"].double()
    p = p - LR * (hat + DECAY * p)
    if case["bits"] == 8 or case["param"] == "bf16":
        k0, k1 = _key(s["seed"], STEP)
        h = torch.arange(n, dtype=torch.int64, device="cuda")
        h = ((h ^ k0) * M1) % 2 ** 32
        h = (((h ^ (h // 2 ** 15)) + k1) * M2) % 2 ** 32
        h = ((h ^ (h // 2 ** 14)) * M3) % 2 ** 32
        h = h ^ (h // 2 ** 16)
    if case["param"] == "bf16":
        ulp = _two(torch.frexp(torch.clamp(p.abs(), min=2.0 ** -126))[1] - 8)
        w = torch.floor(p.abs() / ulp + ((h * M2) % 2 ** 32 // 2 ** 16) / 65536.0) * ulp
        out["param"] = torch.sign(p) * w
    else:
        out["param"] = p
    if case["copy"]:
        out["copy"] = p
    if case["bits"] == 32:
        return {**out, "m": m, "v": v}
    e = _e64(m.abs().view(-1, 128).amax(dim=1))
    lo, step = _grid64((m.abs().view(-1, 128) / _two(e.unsqueeze(1))).view(-1))
    x = (m.abs().view(-1, 128) / _two(e.unsqueeze(1))).view(-1)
    up = (x - lo) / step + ((h // 65536) + 0.5) / 65536.0 >= 1.0
    out["m"], out["m_scale"] = torch.sign(m) * (lo + step * up), _two(e)
    r = torch.sqrt(v)
    e = _e64(r.view(-1, 128).amax(dim=1))
    x = (r.view(-1, 128) / _two(e.unsqueeze(1))).view(-1)
    lo, step = _grid64(x)
    share = (x * x - lo * lo) / ((lo + step) ** 2 - lo * lo)
    q = lo + step * ((h % 65536 + 0.5) / 65536.0 < share)
    out["r"], out["r_scale"] = torch.where(r > 0, torch.clamp(q, min=2.0 ** -9), q), _two(e)
    return out


def exact(case, seed):
    plain = {k: v for k, v in case.items()}
    s = prepare(plain, seed)
    op = case["op"]
    if op == "adamw":
        return _exact_adamw(case, s)
    if op == "norm_forward":
        h = s["x"].double()
        out = {}
        if case["residual"]:
            h = h + s["residual"].double()
            out["h"] = h
            h = h.to(s["x"].dtype).double()      # the sum is kept, and normalised, in the stream's own type
        out["rstd"] = 1.0 / torch.sqrt((h * h).sum(dim=1) / case["cols"] + NORM_EPS)
        out["y"], out["y_scale"], _ = _q64(h * out["rstd"][:, None] * s["weight"].double()[None, :])
        return out
    if op == "norm_backward":
        h, r = s["x"].double(), s["rstd"].double()[:, None]
        dy, w = s["dy"].double(), s["weight"].double()
        inner = (dy * w * h).sum(dim=1, keepdim=True)
        dx = r * dy * w - h * r ** 3 * inner / case["cols"]
        return {"dx": dx + s["dres"].double() if case["residual"] else dx, "dweight": torch.einsum("ij,ij->j", dy, h * r)}
    if op == "quantize":
        x = s["x"].double()
        q, scale, _ = _q64(x)
        qt, scale_t, _ = _q64(x.t().contiguous())
        return {"q": q, "scale": scale, "qt": qt, "scale_t": scale_t}
    M, N, K = case["M"], case["N"], case["K"]
    x = _v64(s["x"], s["x_scale"], K)
    if op == "product":
        return {"y": x @ _v64(s["w"], s["w_scale"], K).t()}
    out = {}
    dy = s["dy"].double()
    out["dyq"], out["dyq_scale"], rows = _q64(dy)
    out["dyt"], out["dyt_scale"], cols = _q64(dy.t().contiguous())
    out["xt"], out["xt_scale"], xt = _q64(x.t().contiguous())
    out["dx"] = rows @ _v64(s["wt"], s["wt_scale"], N).t()
    out["dw"] = s["dw"].double() + cols @ xt.t()
    return out
