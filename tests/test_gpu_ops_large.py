"""Offsets beyond 2^31 elements: the last part of a large tensor against the same values by themselves."""
import pytest
import torch

import paper_2009_02701_b200 as hp

pytestmark = pytest.mark.gpu

U8, BF = torch.uint8, torch.bfloat16


def up(n, a):
    return -(-n // a) * a


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_behind_element_2_to_the_31(bits):
    n, tail = (1 << 31) + 128 * 33 + 37, 128 * 64 + 37
    at = n - tail
    assert at % 128 == 0

    def tensors(k):
        dt = U8 if bits == 8 else torch.float32
        x = dict(param=torch.zeros(k, dtype=BF, device="cuda"), grad=torch.zeros(k, dtype=BF, device="cuda"),
                 m=torch.zeros(k, dtype=dt, device="cuda"), v=torch.zeros(k, dtype=dt, device="cuda"))
        if bits == 8:
            x |= dict(m_scale=torch.zeros(-(-k // 128), dtype=U8, device="cuda"), v_scale=torch.zeros(-(-k // 128), dtype=U8, device="cuda"))
        return x

    g = torch.Generator(device="cuda").manual_seed(1)
    big, small = tensors(n), tensors(tail)
    for name, scale in (("param", 0.1), ("grad", 1e-3)):
        small[name].copy_(torch.randn(tail, generator=g, device="cuda") * scale)
        big[name][at:].copy_(small[name])
    ws = torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8, device="cuda")
    for x, k, offset in ((big, n, 5), (small, tail, 5 + at)):
        table = hp.make_adamw_table([dict(x, n=k, rng_offset=offset, weight_decay=0.1)], hp.HPSGD_BF16, hp.HPSGD_BF16, bits)
        x["norm"] = torch.zeros(2, device="cuda")
        for step in (1, 2):
            hp.hpsgd_grad_norm(table, 0.01, ws, x["norm"])
            hp.hpsgd_adamw_step(table, 1e-3, 0.9, 0.999, 1e-8, step, 7, x["norm"][1:])
    assert torch.allclose(big.pop("norm"), small.pop("norm"), rtol=1e-6)
    if bits == 32:                    # the norms may differ in the last place, and the moments then with them
        assert torch.allclose(big["m"][at:], small["m"], rtol=1e-5, atol=1e-12) and float(big["m"][:at].abs().max()) == 0.0
    for name in ("param", "m_scale", "v_scale"):
        if name in small:
            x = big[name][len(big[name]) - len(small[name]):]
            assert float((x != small[name]).float().mean()) < 1e-3


def test_quantize_and_norm_behind_element_2_to_the_31():
    rows, cols = 70_016, 32_768
    x = torch.zeros(rows, cols, dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    last = torch.randn(128, cols, generator=g, device="cuda").to(BF)
    x[-128:] = last
    q, s = torch.empty(rows, cols, dtype=U8, device="cuda"), torch.empty(cols // 512, rows, 4, dtype=U8, device="cuda")
    qt, st = torch.empty(cols, rows, dtype=U8, device="cuda"), torch.empty(up(rows, 512) // 512, cols, 4, dtype=U8, device="cuda")
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(rows, cols, hp.HPSGD_BF16, x, q=q, scale=s, qt=qt, scale_t=st))
    q1, s1 = torch.empty(128, cols, dtype=U8, device="cuda"), torch.empty(cols // 512, 128, 4, dtype=U8, device="cuda")
    qt1, st1 = torch.empty(cols, 128, dtype=U8, device="cuda"), torch.empty(1, cols, 4, dtype=U8, device="cuda")
    hp.hpsgd_quantize_fp8(hp.make_quantize_fp8(128, cols, hp.HPSGD_BF16, last, q=q1, scale=s1, qt=qt1, scale_t=st1))
    assert torch.equal(q[-128:], q1) and torch.equal(s[:, -128:], s1) and torch.equal(qt[:, -128:], qt1)
    b = rows // 128 - 1
    assert torch.equal(st[b // 4, :, b % 4], st1[0, :, 0])
    # the norm over rows of 16384, of which the last ones lie as far back
    x2 = x.view(rows * 2, cols // 2)
    w = torch.ones(cols // 2, dtype=BF, device="cuda")
    y, y1 = torch.empty_like(x2), torch.empty(256, cols // 2, dtype=BF, device="cuda")
    hp.hpsgd_rmsnorm_forward(hp.make_rmsnorm_forward(rows * 2, cols // 2, 1e-5, hp.HPSGD_BF16, x2, w, y=y))
    hp.hpsgd_rmsnorm_forward(hp.make_rmsnorm_forward(256, cols // 2, 1e-5, hp.HPSGD_BF16, last.view(256, -1), w, y=y1))
    assert torch.equal(y[-256:], y1)


def test_product_with_a_result_behind_element_2_to_the_31():
    M, N, K = 36_000, 60_032, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    a, b = (torch.randint(0, 0x70, (r, K), generator=g, device="cuda", dtype=U8) for r in (M, N))
    sa, sb = (torch.full((1, r, 4), 120, dtype=U8, device="cuda") for r in (M, N))
    d = torch.empty(M, N, dtype=BF, device="cuda")
    hp.hpsgd_gemm_fp8(hp.make_gemm_fp8(M, N, K, a, sa, b, sb, d, hp.HPSGD_BF16))
    t = 300
    d1 = torch.empty(t, N, dtype=BF, device="cuda")
    ws = torch.empty(max(16, hp.hpsgd_gemm_fp8_bytes(t, N, K)), dtype=U8, device="cuda")
    hp.hpsgd_gemm_fp8(hp.make_gemm_fp8(t, N, K, a[-t:].contiguous(), sa[:, -t:].contiguous(), b, sb, d1, hp.HPSGD_BF16, workspace=ws))
    hp.hpsgd_ops_check()
    assert torch.equal(d[-t:], d1)
