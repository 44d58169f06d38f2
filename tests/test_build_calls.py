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
