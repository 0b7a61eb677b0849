"""The operators' refusals: every bad argument is an error code before any GPU work, so all of it runs without a device.
Also the header of the operators: plain C, and what it declares is what is bound and exported."""
import ctypes
import math
import os
import re
import subprocess

import pytest

import paper_2009_02701_b200 as hp
from paper_2009_02701_b200 import binding, build, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "hpsgd_ops.h")
A = 1 << 20            # an address that is aligned for everything; nothing is ever read from it


def refused(code, call, *args, **kw):
    with pytest.raises(hp.HpsgdError) as err:
        call(*args, **kw)
    assert err.value.code == code, str(err.value)


def test_header_declares_what_is_bound_and_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(hpsgd_[a-z_0-9]+)\s*\(", text)))
    lib = ctypes.CDLL(build.build())
    assert names == sorted(ops.SIGNATURES) and all(hasattr(lib, n) for n in names)
    assert not set(names) & set(binding.SIGNATURES)


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "hpsgd_ops.h"\nint probe(void) { hpsgd_adamw_tensor t = {0}; return (int)sizeof t + HPSGD_GRAD_NORM_WORKSPACE + (int)t.n; }\n')
    inc = os.path.join(ROOT, "include")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-fsyntax-only", "-I", inc, str(src)], check=True)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsyntax-only", "-x", "c++", "-I", inc, str(src)], check=True)


def sizeof_in_c(tmp_path, expr):
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include "hpsgd_ops.h"\nint main(void) { printf("%%d", (int)sizeof(%s)); return 0; }\n' % expr)
    exe = tmp_path / "size"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    return int(subprocess.run([str(exe)], capture_output=True, check=True).stdout)


def test_structs_have_the_header_s_size(tmp_path):
    for name in [n for n in dir(ops) if isinstance(getattr(ops, n), type) and issubclass(getattr(ops, n), ctypes.Structure)]:
        assert sizeof_in_c(tmp_path, name) == ctypes.sizeof(getattr(ops, name)), name


# ---------------------------------------------------------------------------------------------- AdamW
ROW = dict(param=A, grad=A, m=A, v=A, n=100)
HY = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)


def table(bits=32, pd=hp.HPSGD_F32, gd=hp.HPSGD_F32, **change):
    return hp.make_adamw_table([{**ROW, **({"m_scale": A, "v_scale": A} if bits == 8 else {}), **change}], pd, gd, bits)


@pytest.mark.parametrize("change", [dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                                    dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=math.nan), dict(step=0),
                                    dict(step=-5), dict(grad_scale=A + 2)], ids=str)
def test_adamw_refuses_hyperparameters(change):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(), **{**HY, **change})


@pytest.mark.parametrize("change", [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1), dict(weight_decay=-0.1),
                                    dict(weight_decay=math.nan), dict(param=A + 2), dict(grad=A + 1), dict(m=A + 2), dict(v=A + 1), dict(copy=A + 1)], ids=str)
def test_adamw_refuses_tensors(change):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(**change), **HY)


def test_adamw_refuses_forms():
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(bits=16), **HY)
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(pd=7), **HY)
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(gd=7), **HY)
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(bits=8, m_scale=None), **HY)
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(bits=8, v_scale=None), **HY)
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_adamw_step, table(pd=hp.HPSGD_BF16, copy=A), **HY)
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_adamw_step, table(n=(1 << 40) + 1), **HY)
    with pytest.raises(TypeError):
        hp.make_adamw_table([{**ROW, "weights": A}], 0, 0, 32)
    lib = hp.load()
    assert lib.hpsgd_adamw_step(None, 1, 0, 0, 32, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None) == hp.HPSGD_E_BADARG
    assert lib.hpsgd_adamw_step(None, -1, 0, 0, 32, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None) == hp.HPSGD_E_BADARG
    assert "n_tensors" in hp.last_error()


@pytest.mark.parametrize("args", [(0.0, A, A), (-1.0, A, A), (math.nan, A, A), (1.0, None, A), (1.0, A + 8, A), (1.0, A, None), (1.0, A, A + 2)], ids=str)
def test_norm_refuses(args):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_grad_norm, table(), *args)
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_grad_norm, table(grad=None), 1.0, A, A)


def test_no_fallback_without_a_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    refused(hp.HPSGD_E_CUDA, hp.hpsgd_adamw_step, table(), **HY)
    refused(hp.HPSGD_E_CUDA, hp.hpsgd_grad_norm, table(), 1.0, A, A)


def test_tables_number_their_random_bits():
    t = hp.make_adamw_table([dict(ROW, n=5), dict(ROW, n=7), dict(ROW, n=1, rng_offset=1 << 40), dict(ROW, n=2)], 0, 0, 32)
    assert [x.rng_offset for x in t.array] == [0, 5, 1 << 40, (1 << 40) + 1]


# ---------------------------------------------------------------------------------------------- norm and quantisation
def norm_args(**change):
    kw = dict(rows=4, cols=256, eps=1e-5, dtype=hp.HPSGD_BF16, x=A, weight=A, residual=A, h=A, y=A, y8=A, y_scale=A, rstd=A)
    return hp.make_rmsnorm_forward(**{**kw, **change})


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=-1), dict(dtype=9), dict(weight_dtype=9), dict(eps=-1.0), dict(eps=math.nan), dict(eps=1e60),
                                    dict(x=None), dict(weight=None), dict(h=None), dict(residual=None), dict(y=None, y8=None, y_scale=None),
                                    dict(y8=None), dict(y_scale=None), dict(x=A + 1), dict(weight=A + 1), dict(rstd=A + 2), dict(h=A + 1), dict(y=A + 1),
                                    dict(y8=A + 8), dict(y_scale=A + 1), dict(ldx=255), dict(ldres=1), dict(ldh=255), dict(ldy=200), dict(ldy8=255),
                                    dict(ldy8=264), dict(ldys=3)], ids=str)
def test_norm_forward_refuses(change):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_rmsnorm_forward, norm_args(**change))


def back_args(**change):
    kw = dict(rows=4, cols=256, dtype=hp.HPSGD_F32, h=A, weight=A, rstd=A, dy=A, dx=A, dweight=A, workspace=A, dres=A)
    return hp.make_rmsnorm_backward(**{**kw, **change})


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=-1), dict(dtype=2), dict(weight_dtype=-1), dict(h=None), dict(weight=None), dict(rstd=None),
                                    dict(dy=None), dict(dx=None), dict(dweight=None), dict(workspace=None), dict(workspace=A + 8), dict(dweight=A + 2),
                                    dict(h=A + 2), dict(dy=A + 1), dict(dres=A + 2), dict(dx=A + 2), dict(ldh=255), dict(lddy=1), dict(lddres=255),
                                    dict(lddx=255)], ids=str)
def test_norm_backward_refuses(change):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_rmsnorm_backward, back_args(**change))


def test_norm_limits():
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_rmsnorm_forward, norm_args(cols=16385))
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_rmsnorm_backward, back_args(cols=16385))
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_rmsnorm_forward, norm_args(rows=1 << 31))
    assert hp.hpsgd_rmsnorm_backward_bytes(10, 100) == 4000 and hp.hpsgd_rmsnorm_backward_bytes(10 ** 6, 100) == 592 * 400
    assert hp.hpsgd_rmsnorm_backward_bytes(0, 100) == 0 and hp.hpsgd_rmsnorm_backward_bytes(5, 20000) == 0
    hp.hpsgd_rmsnorm_forward(norm_args(rows=0))          # nothing to do: no device is asked for
    hp.hpsgd_rmsnorm_backward(back_args(cols=0))
    lib = hp.load()
    for call in (lib.hpsgd_rmsnorm_forward, lib.hpsgd_rmsnorm_backward, lib.hpsgd_quantize_fp8):
        assert call(None, None) == hp.HPSGD_E_BADARG
    with pytest.raises(TypeError):
        norm_args(ldz=5)


def quant_args(**change):
    kw = dict(rows=200, cols=256, dtype=hp.HPSGD_F32, x=A, q=A, scale=A, qt=A, scale_t=A)
    return hp.make_quantize_fp8(**{**kw, **change})


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=-1), dict(dtype=3), dict(x=None), dict(q=None, scale=None, qt=None, scale_t=None), dict(q=None),
                                    dict(scale=None), dict(qt=None), dict(scale_t=None), dict(x=A + 2), dict(q=A + 8), dict(qt=A + 4), dict(scale=A + 1),
                                    dict(scale_t=A + 2), dict(ldx=255), dict(ldq=255), dict(ldq=264), dict(ldqt=200), dict(lds=199), dict(ldst=255),
                                    dict(dtype=hp.HPSGD_FP8, x_scale=A), dict(dtype=hp.HPSGD_FP8, q=None, scale=None),
                                    dict(dtype=hp.HPSGD_FP8, q=None, scale=None, x_scale=A, x=A + 8),
                                    dict(dtype=hp.HPSGD_FP8, q=None, scale=None, x_scale=A, ldx=255),
                                    dict(dtype=hp.HPSGD_FP8, q=None, scale=None, x_scale=A, ldxs=100)], ids=str)
def test_quantize_refuses(change):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_quantize_fp8, quant_args(**change))


def test_quantize_limits():
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_quantize_fp8, quant_args(rows=1 << 31))
    hp.hpsgd_quantize_fp8(quant_args(rows=0))
    hp.hpsgd_quantize_fp8(quant_args(cols=0))


# ---------------------------------------------------------------------------------------------- matrix product
def gemm_args(**change):
    kw = dict(M=300, N=200, K=256, a=A, a_scale=A, b=A, b_scale=A, d=A, d_dtype=hp.HPSGD_F32, workspace=A, workspace_bytes=1 << 30)
    return hp.make_gemm_fp8(**{**kw, **change})


@pytest.mark.parametrize("change", [dict(M=-1), dict(N=-1), dict(K=-1), dict(d_dtype=2), dict(accumulate=2), dict(accumulate=1, d_dtype=hp.HPSGD_BF16),
                                    dict(a=None), dict(b=None), dict(a_scale=None), dict(b_scale=None), dict(d=None), dict(d=A + 2), dict(a=A + 8),
                                    dict(b=A + 8), dict(a_scale=A + 2), dict(b_scale=A + 1), dict(lda=255), dict(lda=264), dict(ldb=240), dict(ldsa=299),
                                    dict(ldsb=199), dict(ldd=199), dict(M=1, K=1 << 17, workspace=None), dict(M=1, K=1 << 17, workspace=A + 8)], ids=str)
def test_product_refuses(change):
    refused(hp.HPSGD_E_BADARG, hp.hpsgd_gemm_fp8, gemm_args(**change))


def test_product_limits():
    refused(hp.HPSGD_E_NOMEM, hp.hpsgd_gemm_fp8, gemm_args(M=1, K=1 << 17, workspace_bytes=100))
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_gemm_fp8, gemm_args(M=1 << 31))
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_gemm_fp8, gemm_args(K=(1 << 31) - 1))
    hp.hpsgd_gemm_fp8(gemm_args(M=0))
    hp.hpsgd_gemm_fp8(gemm_args(N=0))
    assert hp.load().hpsgd_gemm_fp8(None, None) == hp.HPSGD_E_BADARG
    assert hp.hpsgd_gemm_fp8_bytes(0, 5, 5) == 0 and hp.hpsgd_gemm_fp8_bytes(1 << 40, 5, 5) == 0
    # a cluster joins its parts without a workspace; one tile and a very long sum: parts in memory
    assert hp.hpsgd_gemm_fp8_bytes(4096, 4096, 4096) == 0 and hp.hpsgd_gemm_fp8_bytes(1, 128, 1 << 17) > 0
    assert hp.hpsgd_gemm_fp8_bytes(1, 128, 8192) == 0


def test_the_stall_is_for_the_checked_build():
    refused(hp.HPSGD_E_UNSUPPORTED, hp.hpsgd_ops_debug_stall, 1)
