"""The 8-bit layer's operators together, as a training step and a decoding loop use them: forward and backward against 64-bit numbers, on
other streams, from several threads, captured and replayed, and under the range-checked build."""
import json
import os
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

import int8_oracle as O
from paper_2609_26077_b200 import int8

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def inputs(M, N, K, dtype=torch.bfloat16, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g) * torch.exp(torch.randn(K, generator=g))
    return [t.to(dtype).to(device) for t in (x, torch.randn(M, K, generator=g), 1 + 0.2 * torch.randn(K, generator=g),
                                             0.02 * torch.randn(N, K, generator=g), torch.randn(M, N, generator=g), torch.randn(M, K, generator=g))]


def step(x, r, gain, weight, dz, dh, pow2=True):
    """Forward and backward of norm and product; everything a training step would hand on."""
    w, ws = int8.quantize(weight, pow2=pow2)
    n = int8.rms_norm(x, gain, residual=r, pow2=pow2, checkpoint=128)
    z = int8.matmul(n.codes, n.scales, w, ws, dtype=x.dtype)
    dw = int8.grad_weight(dz, n.codes, n.scales)
    dy = int8.grad_input(dz, w, ws)
    dx, dgain = int8.rms_norm_backward(dy, n.checkpoint, n.checkpoint_scales, n.rstd, gain, dresidual=dh)
    return {"w": w, "ws": ws, **n._asdict(), "z": z, "dw": dw, "dy": dy, "dx": dx, "dgain": dgain}


@pytest.mark.parametrize("M,N,K,dtype", [(1, 256, 512, torch.bfloat16), (77, 300, 1000, torch.bfloat16), (515, 1024, 2048, torch.float16),
                                         (2100, 2048, 2304, torch.bfloat16)])
def test_step_against_64_bits(M, N, K, dtype):
    args = inputs(M, N, K, dtype)
    o = step(*args)
    x, r, gain, weight, dz, dh = [O.host(t).astype(np.float64) for t in args]
    u = O.U[dtype]
    h = {k: O.host(v) for k, v in o.items()}
    # what the 8-bit forms stand for is within half a step (and the rounding of the scaling) of what they were taken from
    wv, kv = O.values64(h["w"], h["ws"]), O.values64(h["checkpoint"], h["checkpoint_scales"], 128)
    half = 0.5 + 127 * 2 ** -22
    assert np.all(np.abs(wv - weight) <= half * h["ws"].astype(np.float64)[:, None])
    assert np.all(np.abs(kv - (x + r)) <= half * np.repeat(h["checkpoint_scales"].astype(np.float64), 128, 1)[:, :K] + 2.0 ** -24 * np.abs(x + r))
    rstd = 1 / np.sqrt(((x + r) ** 2).mean(1) + 1e-6)
    nv, y = O.values64(h["codes"], h["scales"]), (x + r) * rstd[:, None] * gain
    assert np.all(np.abs(nv - y) <= half * h["scales"].astype(np.float64)[:, None] + 4 * O.U32 * np.abs(y))
    # the products, from the 8-bit values; power-of-two scales restore exactly in bf16, and in fp16 where they are not subnormal
    z = nv @ wv.T
    O.close(h["z"], z, 4 * O.U32 * np.abs(z) + 1.01 * u * np.abs(z) + O.TINY[dtype])
    slip = 0.0 if dtype is torch.bfloat16 else O.TINY[dtype]
    O.close(h["dw"], dz.T @ nv, M * 2 * O.U32 * (np.abs(dz).T @ np.abs(nv)) + slip * np.abs(dz).sum(0)[:, None] + 1e-37)
    dy = dz @ wv
    O.close(h["dy"], dy, N * 2 * O.U32 * (np.abs(dz) @ np.abs(wv)) + slip * np.abs(dz).sum(1)[:, None] + 1.01 * u * np.abs(dy) + O.TINY[dtype])
    # the norm's gradients, from the dy that was handed on
    dx, size, dgain, gsize = O.rms_norm_backward(h["dy"].astype(np.float64), kv, h["rstd"].astype(np.float64), gain, dh)
    O.close(h["dx"], dx, 100 * O.U32 * size + 1.01 * u * np.abs(dx) + O.TINY[dtype])
    O.close(h["dgain"], dgain, (M + 68) * O.U32 * gsize + 1e-37)


@pytest.mark.parametrize("M,N,K", [(77, 300, 1000), (515, 1024, 2048)])
def test_step_with_default_scales(M, N, K):
    """The step as it is called without options: amax / 127 scales, an fp32 weight gradient, a 16-bit input gradient."""
    args = inputs(M, N, K)
    o = step(*args, pow2=False)
    dz = args[4].double()
    nv, wv = [torch.from_numpy(O.values64(O.host(o[c]), O.host(o[s]))).cuda() for c, s in (("codes", "scales"), ("w", "ws"))]
    assert o["dw"].dtype is torch.float32
    # three parts of every value, a unit of 2^-23 for each addition; the values' rounding to fp32
    want = dz.t() @ nv
    O.close(O.host(o["dw"]), want.cpu().numpy(), ((3 * M + 2) * 2 * O.U32 * (dz.abs().t() @ nv.abs())).cpu().numpy() + 1e-37)
    # an operand of 16 bits would show as up to 2^-8 a value, in the mean 0.0017; the sums' drift is far below 1e-5
    assert ((o["dw"].double() - want).norm() / want.norm()).item() <= 1e-5
    want = dz @ wv
    rounded = (want.bfloat16().double() - want).norm().item()
    assert (o["dy"].double() - want).norm().item() <= 1.03 * rounded


def same(a, b):
    return all(torch.equal(a[k], b[k]) for k in a if isinstance(a[k], torch.Tensor))


@pytest.mark.parametrize("M,N,K", [(5, 200, 600), (1100, 2304, 2048)])
def test_captured_and_replayed(M, N, K):
    """A captured step gives an eager one's bits, on inputs that change between replays, while other calls run in between."""
    first, second = inputs(M, N, K, seed=1), inputs(M, N, K, seed=2)
    want = [step(*a) for a in (first, second)]
    held = [t.clone() for t in first]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(*held)
    torch.cuda.current_stream().wait_stream(s)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:                                   # two graphs of the same calls: workspaces of their own
        with torch.cuda.graph(g):
            outs.append(step(*held))
    for i in (1, 0, 1):
        for t, src in zip(held, (first, second)[i]):
            t.copy_(src)
        graphs[0].replay()
        step(*second)
        graphs[1].replay()
        torch.cuda.synchronize()
        assert same(outs[0], want[i]) and same(outs[1], want[i])
    assert int8.status() == (0, 0)


def test_given_stream_and_given_outputs():
    args = inputs(300, 260, 512, seed=3)
    want = step(*args)
    x, r, gain, weight, dz, dh = args
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = [t.clone() for t in args]               # made on the other stream, used there without a synchronisation
    x, r, gain, weight, dz, dh = late
    w, ws = int8.quantize(weight, pow2=True, stream=s)
    n = int8.rms_norm(x, gain, residual=r, pow2=True, checkpoint=128, hidden=x, stream=s)
    z = int8.matmul(n.codes, n.scales, w, ws, out=torch.empty(300, 260, dtype=torch.bfloat16, device="cuda"), stream=s)
    dw = int8.grad_weight(dz, n.codes, n.scales, out=torch.empty(260, 512, device="cuda"), stream=s)
    dy = int8.grad_input(dz, w, ws, stream=s)
    dx, dgain = int8.rms_norm_backward(dy, n.checkpoint, n.checkpoint_scales, n.rstd, gain, dresidual=dh, dx=dh, stream=s)
    values = int8.dequantize(n.codes, n.scales, stream=s)
    s.synchronize()
    got = {"w": w, "ws": ws, **n._asdict(), "z": z, "dw": dw, "dy": dy, "dx": dx, "dgain": dgain}
    assert same(want, got)
    assert torch.equal(values, int8.dequantize(want["codes"], want["scales"]))
    with pytest.raises(TypeError):
        int8.quantize(torch.zeros(4, 8), stream=s)


def test_two_streams_and_four_threads_at_once():
    cases = [inputs(m, n, k, seed=m) for m, n, k in ((64, 300, 512), (700, 640, 1024), (3, 2048, 2048), (1500, 2304, 512))]
    want = [step(*c) for c in cases]
    torch.cuda.synchronize()
    bad = []

    def run(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = step(*cases[i])
                s.synchronize()
                if not same(got, want[i]):
                    bad.append(i)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    assert int8.status() == (0, 0)


def test_operands_written_just_before_the_call():
    """Every call is ordinary work on the stream: what is before it is complete, what is behind it waits for it."""
    srcs = [inputs(256, 512, 1024, seed=s) for s in (5, 6)]
    want = [step(*a) for a in srcs]
    held = [torch.empty_like(t) for t in srcs[0]]
    got = []
    for i in range(8):
        for t, src in zip(held, srcs[i % 2]):
            torch.mul(src, 1.0, out=t)
        got.append({k: v.clone() for k, v in step(*held).items() if v is not None})
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert same(o, {k: v for k, v in want[i % 2].items() if v is not None})


def test_rows_behind_a_batch_stay_as_they_were():
    """A batch that fills a part of preallocated buffers leaves the rows behind it alone."""
    big = lambda rows, cols, dtype, fill: torch.full((rows, cols), fill, dtype=dtype, device="cuda")
    x, r, gain, weight, dz, dh = inputs(37, 192, 256, seed=8)
    w, ws = int8.quantize(weight)
    codes, scales, out, hidden = big(64, 256, torch.int8, 77), torch.full((64,), -1.0, device="cuda"), big(64, 192, torch.bfloat16, 3.0), big(64, 256, torch.bfloat16, 5.0)
    int8.quantize(x, out=(codes[:37], scales[:37]))
    int8.matmul(codes[:37], scales[:37], w, ws, out=out[:37])
    int8.rms_norm(x, gain, residual=r, hidden=hidden[:37])
    assert (codes[37:] == 77).all() and (scales[37:] == -1).all() and (out[37:] == 3).all() and (hidden[37:] == 5).all()
    assert torch.equal(out[:37], int8.matmul(*int8.quantize(x), w, ws))


def test_offsets_beyond_32_bits():
    """Rows so far apart that elements of one call lie more than 2^32 bytes behind one another."""
    rows, cols, ld = 40, 256, 1 << 27
    store = torch.empty(rows * ld, dtype=torch.int8, device="cuda")
    far = store.view(rows, ld)[:, :cols]
    x = inputs(rows, 8, cols, seed=9)[0]
    scales = torch.empty(rows, device="cuda")
    int8.quantize(x, out=(far, scales))
    codes, want = int8.quantize(x)
    assert torch.equal(far, codes) and torch.equal(scales, want)
    w, ws = int8.quantize(inputs(4, 128, cols, seed=10)[3])
    assert torch.equal(int8.matmul(far, scales, w, ws), int8.matmul(codes, scales, w, ws))
    assert torch.equal(int8.dequantize(far, scales), int8.dequantize(codes, scales))
    dz = torch.randn(rows, 128, device="cuda").bfloat16()
    assert torch.equal(int8.grad_weight(dz, far, scales), int8.grad_weight(dz, codes, scales))
    out = store[: rows * ld].view(torch.bfloat16).view(rows, ld // 2)[:, :128]
    assert torch.equal(int8.matmul(codes, scales, w, ws, out=out), int8.matmul(codes, scales, w, ws))


def test_bounded_wait_is_reported():
    int8.selftest_bounded_wait(1_000_000)
    assert int8.status() == (8, 901)
    int8.status_clear()
    assert int8.status() == (0, 0)
    w, ws = int8.quantize(torch.randn(64, 64, device="cuda"))
    assert torch.isfinite(int8.matmul(w, ws, w, ws)).all()


CHILD = r"""
import json, sys
import torch
sys.path[:0] = [%(root)r, %(root)r + "/tests"]
from paper_2609_26077_b200 import build, fmm
build.build(debug=True)
import test_gpu_int8_layer as T
import test_gpu_int8_product as P
import test_gpu_int8_rows as R
from paper_2609_26077_b200 import int8
assert fmm.lib().fmm_debug_build() == 1
for case in ((1, 256, 512, torch.bfloat16), (77, 300, 1000, torch.bfloat16), (515, 1024, 2048, torch.float16)):
    T.test_step_against_64_bits(*case)
R.test_strides_and_alignment(3, 1)
R.test_norm_backward(torch.float16, 32, True)
R.test_norm_is_bit_exact(torch.bfloat16, True, False, 32)
P.check_matmul(2300, 2100, 256)
P.check_matmul(65, 200, 4095)
P.check_grads(300, 2304, 2200)
P.check_grads(700, 130, 200, dy_extra=3)
print("RESULT", json.dumps(int8.status()))
"""


def test_no_store_outside_its_range():
    r = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT}], capture_output=True, text=True, timeout=900, env=dict(os.environ, FMM_B200_DEBUG="1"))
    assert r.returncode == 0, r.stderr[-3000:]
    line = [ln for ln in r.stdout.splitlines() if ln.startswith("RESULT ")][-1]
    assert json.loads(line[len("RESULT "):]) == [0, 0]
