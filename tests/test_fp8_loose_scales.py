"""CPU checks of scales that lie as any fp32 numbers do, and of a number of tokens that is told: what is refused all the same."""
import ctypes as C

import pytest

from paper_2609_26077_b200 import build as fmm_build
from paper_2609_26077_b200 import fp8

OK, INVALID, SHAPE = 0, 1, 2
P = 4096                    # an address that is never followed: every call here is refused, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    fmm_build.build()
    return fp8.lib()


def filled(kind, base, changes):
    a = kind()
    for k, v in {**base, **changes}.items():
        assert k in dict(kind._fields_)
        setattr(a, k, v)
    return C.byref(a)


def test_quantize(lib):
    base = dict(type=1, scale_mode=0, rows=5, cols=65, x=P, ldx=65, codes=P, ldc=80, scales=P + 4, lds=5, column_codes=P, ldcc=80, column_scales=P + 12, ldcs=65)
    call = lambda **kw: lib.fmm_fp8_quantize(filled(fp8.QuantizeArgs, base, kw), None)
    assert call() == INVALID
    for bad in (dict(scales=P + 2), dict(scales=None), dict(lds=4), dict(column_scales=P + 1), dict(column_scales=None), dict(ldcs=64), dict(ldc=65), dict(ldcc=65)):
        assert call(loose=1, **bad) == INVALID, bad
    assert call(loose=1, rows=0) == OK


@pytest.mark.parametrize("which", ["matmul", "grad_input", "grad_weight"])
def test_products(lib, which):
    M = 128 if which == "grad_weight" else 8
    base = dict(type=0, M=M, N=65, K=33, a=P, lda=80, a_scales=P + 4, lda_scales=65, b=P, ldb=48, b_scales=P + 4, ldb_scales=33, out=P, ldo=65)
    run = getattr(lib, "fmm_fp8_" + which)
    call = lambda **kw: run(filled(fp8.ProductArgs, base, kw), None)
    assert call() == INVALID
    for bad in (dict(a_scales=P + 2), dict(a_scales=None), dict(b_scales=P + 2), dict(b_scales=None), dict(lda_scales=7), dict(lda=65), dict(ldb=33)) + (
            (dict(lda_scales=64), dict(ldb_scales=32)) if which == "grad_weight" else ()):
        assert call(loose=1, **bad) == INVALID, bad
    assert call(loose=1, **dict(matmul=dict(N=0), grad_input=dict(K=0), grad_weight=dict(N=0))[which]) == OK


def test_tokens(lib):
    """The number of tokens that a grouped weight gradient's offsets are cut to."""
    base = dict(type=0, M=256, N=64, K=32, groups=2, offsets=P, a=P, lda=64, a_scales=P, lda_scales=64, b=P, ldb=32, b_scales=P, ldb_scales=32, out=P, ldo=32, step_out=2048)
    call = lambda **kw: lib.fmm_fp8_grad_weight(filled(fp8.ProductArgs, base, kw), None)
    for bad in (-1, 257, 1 << 40):
        assert call(tokens=bad) == SHAPE
    assert call(tokens=200, N=0) == OK
