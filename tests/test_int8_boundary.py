"""CPU checks of the 8-bit integer layer's boundary: every declared function is exported, and unsuitable arguments are refused
on the host, before anything is launched."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2609_26077_b200 import build as fmm_build
from paper_2609_26077_b200 import int8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, SHAPE, WORKSPACE = 0, 1, 2, 4
P = 4096                    # an address that is never followed: every call here is refused, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    fmm_build.build()
    return int8.lib()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "fmm_int8.h")).read()
    declared = set(re.findall(r"\b(fmm_int8_[a-z0-9_]+)\s*\(", text))
    assert declared == set(int8.EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


def filled(kind, base, changes):
    a = kind()
    for k, v in {**base, **changes}.items():
        assert k in dict(kind._fields_)
        setattr(a, k, v)
    return C.byref(a)


def test_quantize_refusals(lib):
    base = dict(x=P, type=0, ldx=64, rows=4, cols=64, block=0, scale_mode=0, codes=P, ldc=64, scales=P)
    call = lambda **kw: lib.fmm_int8_quantize(filled(int8.QuantizeArgs, base, kw), None)
    assert lib.fmm_int8_quantize(None, None) == INVALID
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(type=3), dict(block=64), dict(scale_mode=2), dict(ldx=63), dict(ldc=63),
                dict(x=P + 2), dict(x=P + 1, type=1), dict(scales=P + 2)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=(1 << 31) - 16384, ldx=1 << 31, ldc=1 << 31), dict(cols=1 << 40), dict(rows=(1 << 62) + 1, cols=8)):
        assert call(**bad) == SHAPE, bad
    assert call(rows=0, x=None, codes=None, scales=None) == OK
    assert call(cols=0, block=32, x=None, codes=None, scales=None) == OK


def test_dequantize_refusals(lib):
    base = dict(codes=P, ldc=64, scales=P, rows=4, cols=64, block=0, x=P, type=0, ldx=64)
    call = lambda **kw: lib.fmm_int8_dequantize(filled(int8.DequantizeArgs, base, kw), None)
    assert lib.fmm_int8_dequantize(None, None) == INVALID
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(type=-1), dict(block=16), dict(ldx=63), dict(ldc=63), dict(x=P + 2)):
        assert call(**bad) == INVALID, bad
    assert call(rows=-1) == SHAPE
    assert call(rows=0) == OK and call(cols=0) == OK


def norm_args(**kw):
    a = int8.RmsNormArgs()
    base = dict(type=1, rows=4, cols=64, eps=1e-6, x=P, ldx=64, residual=P, ldr=64, gain=P, hidden=P, ldh=64, codes=P, ldc=64, scales=P,
                rstd=P, checkpoint=P, ldk=64, checkpoint_scales=P, checkpoint_block=32)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def test_rms_norm_refusals(lib):
    call = lambda **kw: lib.fmm_int8_rms_norm(C.byref(norm_args(**kw)), None)
    for bad in (dict(type=5), dict(scale_mode=3), dict(checkpoint_block=64), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(x=None), dict(gain=None), dict(codes=None), dict(scales=None), dict(hidden=None), dict(checkpoint=None), dict(checkpoint_scales=None),
                dict(ldx=63), dict(ldr=63), dict(ldh=63), dict(ldc=63), dict(ldk=63), dict(x=P + 1), dict(gain=P + 1), dict(rstd=P + 2)):
        assert call(**bad) == INVALID, bad
    assert call(rows=-1) == SHAPE and call(cols=1 << 31) == SHAPE
    assert lib.fmm_int8_rms_norm(None, None) == INVALID
    assert call(rows=0, x=None) == OK


def test_rms_norm_backward_refusals(lib):
    def call(ws=P, ws_bytes=1 << 30, **kw):
        a = int8.RmsNormBackwardArgs()
        base = dict(type=1, block=32, rows=4, cols=64, dy=P, ldy=64, checkpoint=P, ldk=64, checkpoint_scales=P, rstd=P, gain=P, dresidual=P,
                    ldr=64, dx=P, ldx=64, dgain=P)
        for k, v in {**base, **kw}.items():
            setattr(a, k, v)
        return lib.fmm_int8_rms_norm_backward(C.byref(a), ws, ws_bytes, None)
    for bad in (dict(type=9), dict(block=1), dict(dy=None), dict(checkpoint=None), dict(checkpoint_scales=None), dict(rstd=None), dict(gain=None),
                dict(dx=None), dict(dgain=None), dict(ldy=63), dict(ldk=63), dict(ldr=63), dict(ldx=63), dict(dgain=P + 2)):
        assert call(**bad) == INVALID, bad
    assert call(rows=-1) == SHAPE
    assert call(ws=None) == WORKSPACE and call(ws=P + 16) == WORKSPACE and call(ws_bytes=63 * 4) == WORKSPACE
    need = C.c_size_t()
    assert lib.fmm_int8_rms_norm_backward_workspace_bytes(4, 64, C.byref(need)) == OK and need.value >= 64 * 4
    assert lib.fmm_int8_rms_norm_backward_workspace_bytes(4, 64, None) == INVALID
    assert lib.fmm_int8_rms_norm_backward_workspace_bytes(-4, 64, C.byref(need)) == SHAPE
    assert call(cols=0, dgain=None) == OK


def test_matmul_refusals(lib):
    base = dict(a=P, lda=64, a_scales=P, b=P, ldb=64, b_scales=P, bias=None, M=4, N=4, K=64, c=P, type=0, ldc=4)
    call = lambda **kw: lib.fmm_int8_matmul(filled(int8.MatmulArgs, base, kw), None)
    assert lib.fmm_int8_matmul(None, None) == INVALID
    for bad in (dict(a=None), dict(b=None), dict(a_scales=None), dict(b_scales=None), dict(c=None), dict(type=3), dict(lda=48), dict(ldb=48), dict(lda=72),
                dict(ldb=72), dict(a=P + 8), dict(b=P + 8), dict(ldc=3), dict(c=P + 2), dict(bias=P + 2), dict(a_scales=P + 2)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(K=131072, lda=131072, ldb=131072), dict(M=1 << 31), dict(N=1 << 33, ldc=1 << 33)):
        assert call(**bad) == SHAPE, bad
    assert call(M=0, a=None, c=None) == OK and call(N=0, b=None, c=None) == OK


@pytest.mark.parametrize("which", ["weight", "input"])
def test_grad_refusals(lib, which):
    base = dict(dy=P, type=1, ldy=64, codes=P, ldc=32, scales=P, M=8, N=64, K=32, out=P, out_type=0, ldo=32)
    run, ask = getattr(lib, f"fmm_int8_grad_{which}"), getattr(lib, f"fmm_int8_grad_{which}_workspace_bytes")
    call = lambda ws=P, ws_bytes=1 << 30, **kw: run(filled(int8.GradArgs, base, kw), ws, ws_bytes, None)
    assert run(None, P, 1 << 30, None) == INVALID
    for bad in (dict(dy=None), dict(codes=None), dict(scales=None), dict(out=None), dict(type=0), dict(out_type=2), dict(ldy=63), dict(ldc=31),
                dict(ldo=31), dict(out=P + 2), dict(dy=P + 1), dict(scales=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(M=-1) == SHAPE and call(N=1 << 31) == SHAPE
    assert call(ws=None) == WORKSPACE and call(ws=P + 128) == WORKSPACE
    need = C.c_size_t()
    sizes = []
    for dy in (P, P + 2):
        assert ask(filled(int8.GradArgs, base, dict(dy=dy)), C.byref(need)) == OK
        assert call(dy=dy, ws_bytes=need.value - 1) == WORKSPACE
        sizes.append(need.value)
    assert sizes[1] > sizes[0] >= 2 * 32 * (8 if which == "weight" else 64)
    assert call(K=0, out=None) == OK
    assert ask(filled(int8.GradArgs, base, {}), None) == INVALID and ask(None, C.byref(need)) == INVALID
    assert ask(filled(int8.GradArgs, base, dict(K=-1)), C.byref(need)) == SHAPE
    # sizes whose workspace no 64 bits hold
    big = dict(M=(1 << 31) - 20000, N=(1 << 31) - 20000, K=(1 << 31) - 20000)
    big.update(ldy=big["N"], ldc=big["K"], ldo=big["K"])
    assert ask(filled(int8.GradArgs, base, big), C.byref(need)) == SHAPE and call(**big) == SHAPE


def test_binding_wants_cuda_tensors_of_the_right_type():
    x = torch.zeros(4, 64)
    codes = torch.zeros(4, 64, dtype=torch.int8)
    s = torch.zeros(4)
    for call in (lambda: int8.quantize(x), lambda: int8.quantize(codes), lambda: int8.dequantize(codes, s), lambda: int8.rms_norm(x, x[0]),
                 lambda: int8.rms_norm_backward(x, codes, s, s, x[0]), lambda: int8.matmul(codes, s, codes, s),
                 lambda: int8.grad_weight(x.bfloat16(), codes, s), lambda: int8.grad_input(x.bfloat16(), codes, s)):
        with pytest.raises((TypeError, ValueError)):
            call()


@pytest.mark.skipif(not os.path.exists(fmm_build.NVCC), reason="nvcc not available")
@pytest.mark.parametrize("source,kernels", [("int8_rows.cu", 50), ("int8_product.cu", 12)])
def test_kernels_have_no_register_spills(source, kernels, tmp_path):
    import subprocess
    assert source in fmm_build.INT8_SOURCES
    cmd = [fmm_build.NVCC] + fmm_build.FLAGS + ["-Xptxas", "-v", "-c", os.path.join(fmm_build.CSRC, source), "-o", str(tmp_path / "o.o")]
    out = subprocess.run(cmd, capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]
    entries = re.findall(r"Compiling entry function '([^']*)'.*?\n.*?\n\s*\d+ bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", out.stderr + out.stdout)
    assert len(entries) >= kernels, "ptxas statistics not found"
    assert not [name for name, st, ld in entries if int(st) or int(ld)]
