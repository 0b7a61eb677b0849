"""What the binding of the operators refuses to take an address of: nothing that a kernel would read or write beyond, in another type, in
another order or in host memory gets as far as a call."""
import numpy as np
import pytest
import torch

import paper_2009_02701_b200 as hp

F32, BF, U8, F16 = torch.float32, torch.bfloat16, torch.uint8, torch.float16
R, C = 24, 200                     # blocks: 2, so one word of scales


def refused(make, *args, **kw):
    with pytest.raises(hp.HpsgdError) as err:
        make(*args, **kw)
    assert err.value.code == hp.HPSGD_E_BADARG
    return str(err.value)


# ---------------------------------------------------------------------------------------------- host memory (needs no device)
@pytest.mark.parametrize("name", ["param", "grad", "m", "v", "m_scale", "v_scale", "copy"])
@pytest.mark.parametrize("host", [torch.zeros(100), np.zeros(100, np.float32), [0.0] * 100], ids=["tensor", "array", "list"])
def test_tables_take_no_host_memory(name, host):
    row = dict(param=1 << 20, grad=1 << 20, m=1 << 20, v=1 << 20, m_scale=1 << 20, v_scale=1 << 20, n=100)
    assert name in refused(hp.make_adamw_table, [{**row, name: host}], hp.HPSGD_F32, hp.HPSGD_F32, 8)


A = 1 << 20
CALLS = {
    "forward": (hp.make_rmsnorm_forward, dict(rows=R, cols=C, eps=1e-5, dtype=0, x=A, weight=A, residual=A, h=A, y=A, y8=A, y_scale=A, rstd=A)),
    "backward": (hp.make_rmsnorm_backward, dict(rows=R, cols=C, dtype=0, h=A, weight=A, rstd=A, dy=A, dx=A, dweight=A, workspace=A, dres=A)),
    "quantize": (hp.make_quantize_fp8, dict(rows=R, cols=C, dtype=0, x=A, q=A, scale=A, qt=A, scale_t=A)),
    "transpose": (hp.make_quantize_fp8, dict(rows=R, cols=C, dtype=hp.HPSGD_FP8, x=A, x_scale=A, qt=A, scale_t=A)),
    "product": (hp.make_gemm_fp8, dict(M=R, N=R, K=C, a=A, a_scale=A, b=A, b_scale=A, d=A, d_dtype=0, workspace=A, workspace_bytes=1 << 20)),
}
POINTERS = [(call, name) for call, (_, kw) in CALLS.items() for name, v in kw.items() if v == A and name != "workspace_bytes"]


@pytest.mark.parametrize("call,name", POINTERS)
def test_arguments_take_no_host_memory(call, name):
    make, kw = CALLS[call]
    make(**kw)                                       # plain addresses are the caller's own affair
    assert name in refused(make, **{**kw, name: torch.zeros(1 << 12)})
    assert name in refused(make, **{**kw, name: np.zeros(1 << 12, np.float32)})


def test_calls_take_no_host_memory():
    table = hp.make_adamw_table([dict(param=A, grad=A, m=A, v=A, n=8)], 0, 0, 32)
    refused(hp.hpsgd_adamw_step, table, 1e-3, 0.9, 0.999, 1e-8, 1, grad_scale=torch.ones(1))
    refused(hp.hpsgd_grad_norm, table, 1.0, torch.zeros(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8), A)
    refused(hp.hpsgd_grad_norm, table, 1.0, A, torch.zeros(2))


# ---------------------------------------------------------------------------------------------- on the device
def z(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def good(call):
    """Tensors that each argument of a call may be."""
    codes, scales = (lambda r, c: z(r, -(-c // 16) * 16, dtype=U8)), (lambda r, c: z(-(-c // 512), r, 4, dtype=U8))
    return {
        "forward": dict(x=z(R, C), residual=z(R, C), h=z(R, C), y=z(R, C), weight=z(C), rstd=z(R), y8=codes(R, C), y_scale=scales(R, C)),
        "backward": dict(h=z(R, C), dy=z(R, C), dx=z(R, C), dres=z(R, C), weight=z(C), rstd=z(R), dweight=z(C), workspace=z(R * C)),
        "quantize": dict(x=z(R, C), q=codes(R, C), scale=scales(R, C), qt=codes(C, R), scale_t=scales(C, R)),
        "transpose": dict(x=codes(R, C), x_scale=scales(R, C), qt=codes(C, R), scale_t=scales(C, R)),
        "product": dict(a=codes(R, C), a_scale=scales(R, C), b=codes(R, C), b_scale=scales(R, C), d=z(R, R), workspace=z(1 << 18)),
    }[call]


@pytest.mark.gpu
@pytest.mark.parametrize("call,name", POINTERS)
def test_wrong_tensors(call, name):
    make, kw = CALLS[call]
    tensors = good(call)
    kw = {**kw, **tensors}
    make(**kw)
    x = tensors[name]
    # memory that ends too early (of operands that are only read, the 8 codes behind the last column need not be there)
    short = z(x.numel() - 9, dtype=x.dtype)
    refused(make, **{**kw, name: short})
    make(**{**kw, name: z(x.numel() + 3, dtype=x.dtype)[3:]})
    if name == "workspace":
        return
    for dtype in (F16, torch.float64, U8 if x.dtype != U8 else F32) + ((BF,) if x.dtype == F32 else ()):
        assert str(dtype) in refused(make, **{**kw, name: z(*x.shape, dtype=dtype)})
    wide = z(*x.shape[:-1], 2 * x.shape[-1], dtype=x.dtype)
    refused(make, **{**kw, name: wide[..., ::2]})                           # elements that are not neighbours
    if x.dim() == 2:
        assert "apart" in refused(make, **{**kw, name: wide[:, : x.shape[-1]]})      # rows further apart than the call is told
        assert "apart" in refused(make, **{**kw, name: z(x.shape[-1], dtype=x.dtype).expand(*x.shape)})


@pytest.mark.gpu
def test_strides_and_leading_dimensions():
    wide = z(R, 3 * C)
    kw = {**CALLS["forward"][1], **good("forward")}
    hp.make_rmsnorm_forward(**{**kw, "x": wide[:, :C]}, ldx=3 * C)
    hp.make_rmsnorm_forward(**{**kw, "x": wide[:, 2 * C:]}, ldx=3 * C)      # the last row ends with its memory
    refused(hp.make_rmsnorm_forward, **{**kw, "x": wide[1:, 2 * C:]}, ldx=3 * C)
    refused(hp.make_rmsnorm_forward, **{**kw, "x": wide[:, :C]}, ldx=2 * C)
    hp.make_rmsnorm_forward(**{**kw, "x": z(2, R // 2, C)})                 # two sequences
    refused(hp.make_rmsnorm_forward, **{**kw, "x": z(R // 2, 2, C).transpose(0, 1)})
    hp.make_rmsnorm_forward(**{**kw, "x": z(R * C)})
    with pytest.raises(TypeError):
        hp.make_rmsnorm_forward(**kw, ldq=C)
    with pytest.raises(TypeError):
        hp.make_quantize_fp8(**CALLS["quantize"][1], ldy=C)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_wrong_tensors_of_a_table(bits):
    n, dt = 300, F32 if bits == 32 else U8
    row = dict(param=z(n), grad=z(n, dtype=BF), m=z(n, dtype=dt), v=z(n, dtype=dt), copy=z(n, dtype=BF), n=n)
    if bits == 8:
        row |= dict(m_scale=z(3, dtype=U8), v_scale=z(3, dtype=U8))
    make = lambda **change: hp.make_adamw_table([{**row, **change}], hp.HPSGD_F32, hp.HPSGD_BF16, bits)  # noqa: E731
    make()
    make(param=z(15, 20), grad=z(n + 5, dtype=BF)[5:])
    for name, x in row.items():
        if name != "n":
            refused(make, **{name: z(x.numel() - 1, dtype=x.dtype)})
            refused(make, **{name: z(*x.shape, dtype=F16)})
            refused(make, **{name: z(2 * x.numel(), dtype=x.dtype)[::2]})
    table = make()
    refused(hp.hpsgd_grad_norm, table, 1.0, z(hp.HPSGD_GRAD_NORM_WORKSPACE - 1, dtype=U8), z(2))
    refused(hp.hpsgd_grad_norm, table, 1.0, z(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8), z(1))
    refused(hp.hpsgd_grad_norm, table, 1.0, z(hp.HPSGD_GRAD_NORM_WORKSPACE, dtype=U8), z(2, dtype=BF))
