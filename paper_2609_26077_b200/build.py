"""Build the CUDA library in-tree: paper_2609_26077_b200/libfmm_b200.so (sm_100a only), the Python module _calls that calls it for the usual
arguments (csrc/calls.cpp, against the installed torch, which its file name tells), and on request the library's checked twin libfmm_b200_debug.so (-DFMM_DEBUG: every global store of every kernel is range-checked)."""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libfmm_b200.so")
SOURCES = ["fmm_api.cu", "fmm_encode.cu", "fmm_gemm.cu", "fmm_keep.cu", "fmm_split.cu", "fmm_stats.cu"]
INT8_SOURCES = ["int8_rows.cu", "int8_product.cu"]          # the 8-bit integer layer (include/fmm_int8.h), in the same library
FP8_SOURCES = ["fp8_rows.cu", "fp8_product.cu"]             # the 8-bit floating-point layer (include/fmm_fp8.h)
GRADIENT_SOURCES = ["gradients.cu"]                         # norm and clipping of all gradients (include/fmm_gradients.h)
HEADERS = [os.path.join(CSRC, h) for h in sorted(os.listdir(CSRC)) if h.endswith((".h", ".cuh"))] + [
    os.path.join(HERE, "..", "include", h) for h in ("fmm.h", "fmm_int8.h", "fmm_fp8.h", "fmm_gradients.h")]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-cudart", "static"]


CALLS_SOURCE = os.path.join(CSRC, "calls.cpp")
OUT_DEBUG = os.path.join(HERE, "libfmm_b200_debug.so")


def _stale(out):
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    deps = [os.path.join(CSRC, s) for s in SOURCES + INT8_SOURCES + FP8_SOURCES + GRADIENT_SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def calls_path() -> str:
    """The module for the installed torch and this Python.  It knows how their objects lie in memory, so its name says which ones it was built against: that of
    another torch is another file, and is not loaded."""
    import torch
    version = f"{torch.__version__}-{(torch.version.git_version or '')[:8]}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}"
    return os.path.join(HERE, f"_calls.torch-{version}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_calls(force: bool = False) -> str:
    out = calls_path()
    headers = [h for h in HEADERS if h.endswith(("fmm.h", "fmm_int8.h", "fmm_fp8.h", "fmm_gradients.h"))]
    if not force and os.path.exists(out) and all(os.path.getmtime(d) <= os.path.getmtime(out) for d in [CALLS_SOURCE] + headers):
        return out
    import torch
    at = os.path.dirname(torch.__file__)
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for include in (os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"],
                    os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")):
        cmd += ["-isystem", include]
    part = f"{out}.{os.getpid()}.so"                          # (a process that loads the module meanwhile sees the old one or the new one)
    try:
        subprocess.check_call(cmd + [CALLS_SOURCE, "-o", part, "-L" + os.path.join(at, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch", "-ltorch_python"])
        os.replace(part, out)
    finally:
        if os.path.exists(part):
            os.remove(part)
    return out


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """The library, which needs nvcc alone, and the module, where torch and a compiler for it are there."""
    out = build_library(force, verbose, debug)
    try:
        build_calls(force)
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        print(f"the module for the usual calls is not built: {e}", file=sys.stderr)
    return out


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    out = OUT_DEBUG if debug else OUT
    if not force and not _stale(out):
        return out
    objs = []
    procs = []
    for s in SOURCES + INT8_SOURCES + FP8_SOURCES + GRADIENT_SOURCES:
        o = os.path.join(CSRC, s.replace(".cu", ".dbg.o" if debug else ".o"))
        cmd = ([NVCC] + FLAGS + (["-DFMM_DEBUG"] if debug else []) + (["-Xptxas", "-v"] if verbose else []) +
               ["-c", os.path.join(CSRC, s), "-o", o])
        procs.append((subprocess.Popen(cmd), cmd))
        objs.append(o)
    for p, cmd in procs:
        if p.wait() != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    subprocess.check_call([NVCC, "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a",
                           "-o", out] + objs)
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
