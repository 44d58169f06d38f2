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
