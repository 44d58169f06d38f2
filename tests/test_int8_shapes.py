"""Launch rules of the 8-bit layer's row kernels (csrc/int8_shapes.h, plain C++, compiled here): the kernels that test nothing are taken
for rows that fill every thread, and for no others."""
import ctypes as C
import shutil
import subprocess

import pytest

from paper_2609_26077_b200 import build as B

CXX = shutil.which("g++") or shutil.which("c++")
pytestmark = pytest.mark.skipif(CXX is None, reason="no C++ compiler")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("shapes")
    src, so = tmp / "shapes.cpp", tmp / "shapes.so"
    src.write_text('#include "int8_shapes.h"\n'
                   'extern "C" void row_form(long long cols, int* out)\n'
                   '{ const Int8RowForm f = int8_row_form(cols); out[0] = f.vpt; out[1] = f.threads; out[2] = f.whole; }\n')
    subprocess.check_call([CXX, "-O2", "-std=c++17", "-shared", "-fPIC", "-I", B.CSRC, str(src), "-o", str(so)])
    return C.CDLL(str(so))


def row_form(lib, cols):
    out = (C.c_int * 3)()
    lib.row_form(C.c_longlong(cols), out)
    return out[0], out[1], bool(out[2])


def test_untested_kernels_have_a_column_for_every_thread(lib):
    for cols in list(range(0, 20000)) + [(1 << 31) - 16385]:
        vpt, threads, whole = row_form(lib, cols)
        assert vpt in (2, 4) and threads % 32 == 0
        assert threads * vpt * 8 >= cols > (threads - 32) * vpt * 8 or cols == 0
        # what the kernels without tests read and write is threads x vpt x 8 columns, and at least a warp's
        assert whole == (cols > 0 and cols == max(threads, 32) * vpt * 8), cols


def test_rows_without_columns_take_no_untested_kernel(lib):
    assert not row_form(lib, 0)[2]


def test_product_shapes_are_refused_on_the_host():
    B.build()
    from paper_2609_26077_b200 import int8
    lib, s = int8.lib(), int8.ProductShape()
    ask = lambda *a: lib.fmm_int8_product_shape(*a, C.byref(s))
    assert lib.fmm_int8_product_shape(0, 1, 1, 1, 0, None) == 1
    for bad in ((3, 1, 1, 1, 0), (-1, 1, 1, 1, 0), (0, 1, 1, 1, 3)):
        assert ask(*bad) == 1, bad
    for bad in ((0, 0, 1, 1, 0), (0, 1, 1, 131072, 0), (1, 1, 0, 1, 0), (2, 1, 1, 1 << 31, 0), (0, 1 << 31, 1, 1, 0)):
        assert ask(*bad) == 2, bad
    for form in ((1, 256, 1), (2, 16, 8), (3, 8, 1)):
        assert lib.fmm_int8_force_product_shape(C.byref(int8.ProductShape(*form))) == 0
        assert ask(0, 5, 5, 5, 0) == 0 and tuple(s) == form
    for form in ((0, 0, 0), (1, 256, 2), (2, 16, 9), (2, 256, 1), (3, 16, 1)):
        assert lib.fmm_int8_force_product_shape(C.byref(int8.ProductShape(*form))) == 1
        assert ask(0, 5, 5, 5, 0) == 0 and tuple(s) == (3, 8, 1)
    assert lib.fmm_int8_force_product_shape(None) == 0
