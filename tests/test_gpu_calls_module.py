"""What the module _calls does around the library's entry points: other Python threads run meanwhile, and a call that failed is not made again."""
import ctypes as C
import subprocess
import threading
import time

import pytest
import torch

from paper_2609_26077_b200 import fmm, fp8, gradients

pytestmark = pytest.mark.gpu

ENTRIES = ["fmm_fp8_quantize", "fmm_fp8_matmul", "fmm_fp8_grad_input", "fmm_fp8_grad_weight", "fmm_gradient_workspace_bytes", "fmm_gradient_norm", "fmm_gradient_clip"]
CUDA_ERROR = 6

SOURCE = r"""
#include <unistd.h>
int calls = 0;
int slow(void) { ++calls; usleep(400000); return 1; }        /* an argument that the library refuses, after a while */
int fails(void) { ++calls; return %d; }                      /* an error of the device, after whatever was enqueued */
""" % CUDA_ERROR


@pytest.fixture
def bound(tmp_path):
    """bind(name): every entry point but that for the workspace's size is the function of that name; its count of calls."""
    (tmp_path / "entries.c").write_text(SOURCE)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(tmp_path / "entries.so"), str(tmp_path / "entries.c")])
    other, lib = C.CDLL(str(tmp_path / "entries.so")), fp8.lib()
    address = lambda f: C.cast(f, C.c_void_p).value
    real = [address(getattr(lib, name)) for name in ENTRIES]
    calls = C.c_int.in_dll(other, "calls")

    def bind(name):
        fp8._usual().bind(*(real[i] if "workspace" in n else address(getattr(other, name)) for i, n in enumerate(ENTRIES)))
        calls.value = 0
        return calls
    yield bind
    fp8._usual().bind(*real)


def usual_calls():
    """Each kind of call that the module makes, and what it may write to."""
    x, dy = torch.randn(40, 200, device="cuda"), torch.randn(40, 72, device="cuda")
    w = fp8.quantize_weight(torch.randn(72, 200, device="cuda"))
    q, g = fp8.quantize_both(x), fp8.quantize_both(dy)
    y, dx, dw, grad = (torch.ones(*s, device="cuda") for s in ((40, 72), (40, 200), (72, 200), (100,)))
    torch.cuda.synchronize()
    return [(lambda: fp8.quantize(x), None), (lambda: fp8.matmul(q.codes, q.scales, *w, out=y), y), (lambda: fp8.grad_input(g.codes, g.scales, *w, out=dx, accumulate=True), dx),
            (lambda: fp8.grad_weight(g.column_codes, g.column_scales, q.column_codes, q.column_scales, out=dw, accumulate=True), dw), (lambda: gradients.norm([grad]), None),
            (lambda: gradients.clip([grad], 0.5), grad)]


def test_other_threads_run_meanwhile(bound):
    """A launch may wait for the device, and what the device waits for may be another thread's to do."""
    calls = usual_calls()
    count = bound("slow")
    for call, _ in calls:
        ticks, stop = [], threading.Event()

        def tick():
            while not stop.is_set():
                ticks.append(time.monotonic())
                time.sleep(0.002)
        thread = threading.Thread(target=tick)
        thread.start()
        while not ticks:
            time.sleep(0.001)
        count.value = 0
        start = time.monotonic()
        call()                                               # refused after 0.4 s; the general way, which has the real entries, does it then
        stop.set()
        thread.join()
        assert count.value == 1
        # (a thread that holds on to the interpreter for the whole of the 0.4 s leaves none)
        assert len([t for t in ticks if start + 0.05 < t < start + 0.35]) >= 10


def test_a_call_that_failed_is_not_made_again(bound):
    """Its work may have been enqueued: once more would add or scale twice."""
    calls = usual_calls()
    for call, out in calls:
        before = None if out is None else out.clone()
        count = bound("fails")
        with pytest.raises(fmm.FmmError):
            call()
        assert count.value == 1
        assert out is None or torch.equal(out, before)


def test_refusals_still_go_the_general_way():
    t = torch.ones(64, device="cuda")
    with pytest.raises(fmm.FmmError, match="fmm_gradient_clip"):
        gradients.clip([t, t], 1.0)
    assert (t == 1).all()


def test_without_the_module_the_general_way_does_it(monkeypatch, tmp_path):
    x, w = torch.randn(40, 200, device="cuda"), fp8.quantize_weight(torch.randn(72, 200, device="cuda"))
    step = lambda: (*(t.view(torch.uint8) for t in fp8.quantize(x)), fp8.matmul(*fp8.quantize(x), *w), gradients.norm([x]), gradients.clip([x], 1.0, out=[torch.empty_like(x)]))
    want = step()
    monkeypatch.setattr(fp8.build, "calls_path", lambda: str(tmp_path / "_calls.so"))
    monkeypatch.setattr(fp8, "_lib", None)
    monkeypatch.setattr(fp8, "_calls", None)
    with pytest.warns(RuntimeWarning, match="through ctypes"):
        got = step()
    assert fp8._usual().quantize(x, None, False, 1) is None
    assert all(torch.equal(a, b) for a, b in zip(got, want))
