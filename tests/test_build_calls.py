"""The module that makes the usual calls from Python is built against the installed torch; the library needs nvcc alone."""
import os
import subprocess
import sys

import pytest

from paper_2609_26077_b200 import build as fmm_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code, **env):
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, env=dict(os.environ, **env))
    assert r.returncode == 0, r.stderr[-2000:]
    return r


@pytest.mark.parametrize("lacking,env", [("sys.modules['torch'] = None", {}), ("", {"CXX": "/bin/false"}), ("", {"CXX": "/no/such/compiler"})])
def test_library_without_torch_or_its_compiler(lacking, env, tmp_path):
    fmm_build.build()
    newer = tmp_path / "calls.cpp"                           # so that the module has to be built again
    newer.write_text("#error not to be compiled")
    r = run(f"import sys\n{lacking}\n" + f"""
from paper_2609_26077_b200 import build
build.CALLS_SOURCE = {str(newer)!r}
assert build.build() == build.OUT
""", **env)
    assert "is not built" in r.stderr


def test_module_is_that_of_the_torch_that_is_there():
    """Another torch or Python, another file: one that was built against another is neither taken for up to date nor loaded."""
    import torch
    fmm_build.build()
    path = fmm_build.calls_path()
    assert os.path.exists(path) and torch.__version__ in path and f"{sys.version_info[0]}{sys.version_info[1]}" in os.path.basename(path)
    r = run("""
import torch
from paper_2609_26077_b200 import build
before = build.calls_path()
torch.__version__ = "9.9.9"
assert build.calls_path() != before and not build.os.path.exists(build.calls_path())
torch.__version__, torch.version.git_version = "%s", "another"
assert build.calls_path() != before
build.sysconfig.get_config_var = lambda name: ".cpython-399-x86_64-linux-gnu.so"
assert build.calls_path() != before
""" % torch.__version__)


@pytest.mark.parametrize("what", ["nothing", "no module"])
def test_calls_without_the_module(what, tmp_path):
    """A warning, and the general way for every call."""
    path = tmp_path / "_calls.so"
    if what == "no module":
        path.write_text("neither")
    r = run(f"""
import warnings
from paper_2609_26077_b200 import build, fp8, gradients
build.calls_path = lambda: {str(path)!r}
with warnings.catch_warnings(record=True) as seen:
    warnings.simplefilter("always")
    fp8.lib(), gradients.lib(), fp8.lib()
assert [w.category for w in seen] == [RuntimeWarning] and "through ctypes" in str(seen[0].message)
import torch
x = torch.zeros(4, 4)
for call in (lambda: fp8.quantize(x), lambda: fp8.matmul(x, x, x, x), lambda: fp8.grad_weight(x, x, x, x), lambda: gradients.norm([x]), lambda: gradients.clip([x], 1.0)):
    try:
        call()
    except TypeError as e:
        assert "CUDA tensor" in str(e)
    else:
        raise AssertionError
""")
