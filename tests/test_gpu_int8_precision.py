"""How exactly the gradients of the 8-bit product hold what the 8-bit forms stand for: fp32 gradients in fp32 whatever the scales, 16-bit
ones up to their own rounding, fp16 values without leaving its range."""
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
from test_gpu_int8_product import codes_of, padded, scales_of

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAX_PARTS = 3


def cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def poison_free_memory():
    """Memory that the next allocations get holds NaN in every type."""
    held = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in (1 << 26, 1 << 24, 1 << 22, 1 << 20, 1 << 18)]
    torch.cuda.synchronize()
    del held


def values(codes, scales):
    return cuda(codes).double() * cuda(scales).double()[:, None]


def grads(dy, x, sx, w, sw, out_type):
    poison_free_memory()
    dw = int8.grad_weight(dy, padded(x), cuda(sx), dtype=out_type)
    poison_free_memory()
    return dw, int8.grad_input(dy, padded(w), cuda(sw), dtype=out_type)


def exact_grads(dy, x, sx, w, sw):
    """Both gradients in 64 bits, and the sums of their terms' magnitudes."""
    d, vx, vw = dy.double(), values(x, sx), values(w, sw)
    return d.t() @ vx, d.abs().t() @ vx.abs(), d @ vw, d.abs() @ vw.abs()


def spread_scales(rows, seed, lo=-20, hi=6):
    """Scales over many powers of two; of every other 64 rows powers of two, of the others one that is none at least."""
    g = np.random.default_rng([seed, 2])
    s = np.exp2(g.integers(lo, hi, rows)).astype(np.float32)
    other = np.arange(rows) // 64 % 2 == 1
    s[other] *= (1 + g.random(int(other.sum()))).astype(np.float32)
    return s


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scales", ["default", "mixed"])
@pytest.mark.parametrize("M,N,K", [(1, 3, 7), (64, 130, 200), (65, 63, 129), (300, 290, 257), (200, 300, 2500), (300, 3000, 1000)])
def test_fp32_gradients_are_fp32(M, N, K, scales, dtype):
    make = scales_of if scales == "default" else spread_scales
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(M)).to(dtype).cuda()
    x, w = codes_of(M, K, 1), codes_of(N, K, 2)
    sx, sw = make(M, 3), make(N, 4)
    if N > 300:
        sw = scales_of(N, 4, pow2=True)         # (a long contraction's bound would not tell 16 bits from 32)
    dw, dx = grads(dy, x, sx, w, sw, torch.float32)
    want_w, size_w, want_x, size_x = exact_grads(dy, x, sx, w, sw)
    # a unit of 2^-23 for each addition of a product's parts; the values: rounded to fp32 (2^-24) and, of fp16, to two parts (2^-21, or 2^-25
    # where the largest scale lies in [128, 256))
    for got, want, size, n, s in ((dw, want_w, size_w, M, sx), (dx, want_x, size_x, N, sw)):
        bound = (MAX_PARTS * n + 2) * 2 * O.U32 * size + 1e-37
        if dtype is torch.float16:
            bound = bound + 2.0 ** -25 * 2.0 ** -6 * float(s.max()) * (dy.double().abs().sum(0)[:, None] if got is dw else dy.double().abs().sum(1)[:, None])
        O.close(O.host(got), want.cpu().numpy(), bound.cpu().numpy())


def rounding(want, dtype):
    return (want.to(dtype).double() - want).norm().item()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", [(257, 512, 1000), (1001, 2048, 2047), (130, 4100, 1100), (2304, 2560, 2304)])
def test_16_bit_gradients_up_to_their_rounding(M, N, K, dtype):
    """Default scales.  The output's own rounding is all that shows: with an operand rounded to the same type the error is sqrt(2) times it.
    (dY * scale in fp16 is off by an eighth of bf16's rounding, which adds in squares: 1.008.)"""
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(N)).to(dtype).cuda()
    x, w, sx, sw = codes_of(M, K, 1), codes_of(N, K, 2), scales_of(M, 3), scales_of(N, 4)
    sx, sw = sx / 16, sw / 16                   # (inside half precision's range)
    dw, dx = grads(dy, x, sx, w, sw, dtype)
    want_w, _, want_x, _ = exact_grads(dy, x, sx, w, sw)
    for got, want in ((dw, want_w), (dx, want_x)):
        assert got.dtype is dtype
        assert (got.double() - want).norm().item() <= 1.03 * rounding(want, dtype)


@pytest.mark.parametrize("out_type", [torch.float32, torch.float16])
def test_fp16_values_stay_in_range(out_type):
    """fp16 activations at the type's limit: with power-of-two scales 65504 is held as 64 * 1024, which fp16 does not have."""
    M, N, K = 96, 40, 72
    g = torch.Generator().manual_seed(1)
    x = (torch.rand(M, K, generator=g) * 2 - 1).half()
    x[::3, 5] = 65504
    x[1::3] *= 2.0 ** -13                       # and rows of subnormal numbers
    dy = (torch.randn(M, N, generator=g) * 2.0 ** -12).half().cuda()
    for pow2 in (True, False):
        codes, scales = int8.quantize(x.cuda(), pow2=pow2)
        if pow2:
            assert (codes.float() * scales[:, None]).abs().max() > 65504
        v = codes.double() * scales.double()[:, None]
        poison_free_memory()
        got = int8.grad_weight(dy, codes, scales, dtype=out_type)
        want, size = dy.double().t() @ v, dy.double().abs().t() @ v.abs()
        assert torch.isfinite(got.float()).all()
        bound = (MAX_PARTS * M + 2) * 2 * O.U32 * size + 1.01 * O.U[out_type] * want.abs() + O.TINY[out_type]
        bound = bound + 2.0 ** -25 * 2.0 ** -6 * scales.max().double() * dy.double().abs().sum(0)[:, None]
        O.close(O.host(got), want.cpu().numpy(), bound.cpu().numpy())


def test_input_gradient_of_rows_far_apart():
    """Rows of dY, and numbers within a row, over the range that bf16 has; weights with scales far apart."""
    M, N, K = 70, 200, 90
    g = np.random.default_rng(5)
    dy = torch.from_numpy(g.standard_normal((M, N)) * np.exp2(g.integers(-18, 1, (M, N)).astype(np.float64)) * np.exp2(np.linspace(-90, 90, M))[:, None]).bfloat16().cuda()
    dy[3] = 0
    w, sw = codes_of(N, K, 2), spread_scales(N, 6, -10, 4)
    for offset in (0, 1):
        dyc = O.strided(dy, 3, offset) if offset else dy
        poison_free_memory()
        dx = int8.grad_input(dyc, padded(w), cuda(sw))
        v = values(w, sw)
        want, size = dy.double() @ v, dy.double().abs() @ v.abs()
        # dY * scale rounded to fp32 and fp16, or to 2^-25 of a unit that is 2^-15 of the row's largest; the sums; the output
        floor = (dy.double() * cuda(sw).double()).abs().max(1).values[:, None] * 2.0 ** -39 * cuda(w).double().abs().sum(0)
        bound = (2.0 ** -11 + (N + 2) * 2 * O.U32) * size + floor + 1.01 * O.U[torch.bfloat16] * want.abs() + O.TINY[torch.bfloat16]
        O.close(O.host(dx), want.cpu().numpy(), bound.cpu().numpy())
        assert not dx[3].any()


@pytest.mark.parametrize("dtype,out_type", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16)])
def test_infinities_and_nan_go_where_they_belong(dtype, out_type):
    """As in the products of the values: a NaN or an infinity of dY, and a block without a scale, reach what they are a term of."""
    M, N, K = 140, 200, 150
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).to(dtype)
    dy[5, 7], dy[70, 100], dy[71, 3] = float("nan"), float("inf"), float("-inf")
    dy = dy.cuda()
    for pow2 in (True, False):
        x, w, sx, sw = codes_of(M, K, 1), codes_of(N, K, 2), scales_of(M, 3, pow2), scales_of(N, 4, pow2)
        x[70, 11] = w[100, 13] = 0
        for bad in (False, True):
            if bad:
                sx[20], sw[30] = np.nan, np.nan
            dw, dx = grads(dy, x, sx, w, sw, out_type)
            want_w, _, want_x, _ = exact_grads(dy, x, sx, w, sw)
            for got, want in ((dw, want_w), (dx, want_x)):
                assert torch.equal(torch.isnan(got), torch.isnan(want))
                assert torch.equal(torch.isposinf(got), torch.isposinf(want)) and torch.equal(torch.isneginf(got), torch.isneginf(want))
                assert bad or torch.isfinite(got).any()


def test_gradients_add_to_what_is_there():
    M, N, K = 130, 200, 260
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    w, sw = codes_of(N, K, 2), scales_of(N, 4)
    old = torch.randn(M, K, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    got = int8.grad_input(dy, padded(w), cuda(sw), out=old.clone(), accumulate=True)
    want = dy.double() @ values(w, sw) + old.double()
    assert (got.double() - want).norm().item() <= 1.03 * rounding(want, torch.bfloat16)


@pytest.mark.parametrize("dtype,out_type", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float16, torch.float32)])
def test_rounded_values_on_request(dtype, out_type):
    """rounded=True: every value rounded once to dY's type, whatever the scales; a workspace of its own size."""
    M, N, K = 300, 290, 257
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    x, w, sx, sw = codes_of(M, K, 1), codes_of(N, K, 2), scales_of(M, 3), scales_of(N, 4)
    for rounded in (True, False, True):
        dw = int8.grad_weight(dy, padded(x), cuda(sx), dtype=out_type, rounded=rounded)
        dx = int8.grad_input(dy, padded(w), cuda(sw), dtype=out_type, rounded=rounded)
        if rounded:
            d, vx, vw = dy.double(), values(x, sx), values(w, sw)
            # (the fp16 values' power of two moves their rounding only where they are subnormal without it)
            rx, rw = vx.float().to(dtype).double(), vw.float().to(dtype).double()
            for got, want, size, n in ((dw, d.t() @ rx, d.abs().t() @ rx.abs(), M), (dx, d @ rw, d.abs() @ rw.abs(), N)):
                bound = n * 2 * O.U32 * size + O.U[out_type] * want.abs() * 1.01 + O.TINY[out_type]
                if dtype is torch.float16:
                    bound = bound + 2.0 ** -25 * 1.01 * (d.abs().sum(0)[:, None] if got is dw else d.abs().sum(1)[:, None])
                O.close(O.host(got), want.cpu().numpy(), bound.cpu().numpy())


# ------------------------------------------------------------------------------------------------ the chains of kernels
CHAINS = [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.float16, torch.float16)]


def both(dy, x, sx, w, sw, out_type, **how):
    return int8.grad_weight(dy, x, sx, dtype=out_type, **how), int8.grad_input(dy, w, sw, dtype=out_type, **how)


def case(M, N, K, dtype, seed, pow2=False, dy_offset=0):
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()
    return [O.strided(dy, 3, dy_offset) if dy_offset else dy, padded(codes_of(M, K, seed)), cuda(scales_of(M, seed, pow2)),
            padded(codes_of(N, K, seed + 1)), cuda(scales_of(N, seed + 1, pow2))]


@pytest.mark.parametrize("M,N,K,dy_offset", [(300, 520, 384, 0), (300, 520, 384, 1), (2200, 4200, 130, 0), (40, 8200, 72, 1)])
@pytest.mark.parametrize("dtype,out_type", CHAINS)
def test_captured_and_replayed(dtype, out_type, M, N, K, dy_offset):
    """Two graphs of the same calls, replayed on inputs that change in between (default scales, powers of two, others), eager calls on the same
    stream between them: the bits of eager calls."""
    sources = [case(M, N, K, dtype, 1, False, dy_offset), case(M, N, K, dtype, 2, True, dy_offset), case(M, N, K, dtype, 3, False, dy_offset)]
    want = [both(*c, out_type) for c in sources]
    held = case(M, N, K, dtype, 4, False, dy_offset)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(*held, out_type)
    torch.cuda.current_stream().wait_stream(s)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(both(*held, out_type))
    for i in (0, 1, 2, 0):
        for t, src in zip(held, sources[i]):
            t.copy_(src)
        graphs[0].replay()
        both(*sources[1], out_type)
        graphs[1].replay()
        torch.cuda.synchronize()
        for got in outs:
            assert torch.equal(got[0], want[i][0]) and torch.equal(got[1], want[i][1])
    assert int8.status() == (0, 0)


def test_threads_and_streams_at_once():
    cases = [(case(300 + 64 * i, 520, 384 + 8 * i, dtype, i, pow2, offset), out_type)
             for i, ((dtype, out_type), pow2, offset) in enumerate(zip(CHAINS, (False, True, False, False), (0, 1, 1, 0)))]
    want = [both(*c, t) for c, t in cases]
    torch.cuda.synchronize()
    bad = []

    def run(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(30):
                got = both(*cases[i][0], cases[i][1])
                s.synchronize()
                if not (torch.equal(got[0], want[i][0]) and torch.equal(got[1], want[i][1])):
                    bad.append(i)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad and int8.status() == (0, 0)


def test_alignment_of_dy_leaves_no_trace():
    for dtype, out_type in CHAINS:
        aligned = case(140, 203, 150, dtype, 5)
        want = both(*aligned, out_type)
        for extra, offset in ((3, 1), (5, 2), (8, 0)):
            got = both(O.strided(aligned[0], extra, offset), *aligned[1:], out_type)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("M,N,K", [(3, 16424, 24), (1190, 16424, 24), (1201, 8200, 24), (700, 8192, 40), (700, 5000, 33), (2500, 300, 16)])
def test_rows_of_dy_of_every_length(M, N, K):
    """A warp to a block a row, rows that fit registers and rows that do not, few of them and many, aligned and not."""
    dy, _, _, w, sw = case(M, N, K, torch.bfloat16, 6)
    v = w.double() * sw.double()[:, None]
    want, size = dy.double() @ v, dy.double().abs() @ v.abs()
    floor = (dy.double() * sw.double()).abs().max(1).values[:, None] * 2.0 ** -39 * w.double().abs().sum(0)
    # sums of at most 8192 terms leave the accumulator, three more additions
    bound = (2.0 ** -11 + (min(N, 8192) + 4) * 2 * O.U32) * size + floor + 1.01 * O.U[torch.bfloat16] * want.abs()
    for offset in (0, 1):
        poison_free_memory()
        dx = int8.grad_input(O.strided(dy, 3, offset) if offset else dy, w, sw)
        O.close(O.host(dx), want.cpu().numpy(), bound.cpu().numpy())
        assert (dx.double() - want).norm() <= 1.03 * (want.bfloat16().double() - want).norm()


CHILD = r"""
import json, sys
import torch
sys.path[:0] = [%(root)r, %(root)r + "/tests"]
from paper_2609_26077_b200 import build, fmm, int8
build.build(debug=True)
import test_gpu_int8_forms as F
import test_gpu_int8_precision as P
import test_gpu_int8_rows as R
assert fmm.lib().fmm_debug_build() == 1
P.test_fp32_gradients_are_fp32(65, 63, 129, "mixed", torch.float16)
P.test_fp32_gradients_are_fp32(300, 290, 257, "default", torch.bfloat16)
P.test_16_bit_gradients_up_to_their_rounding(257, 512, 1000, torch.bfloat16)
P.test_16_bit_gradients_up_to_their_rounding(257, 512, 1000, torch.float16)
P.test_alignment_of_dy_leaves_no_trace()
P.test_rows_of_dy_of_every_length(1190, 16424, 24)
P.test_rows_of_dy_of_every_length(3, 16424, 24)
P.test_rows_of_dy_of_every_length(700, 5000, 33)
R.test_rows_without_columns_touch_nothing(torch.bfloat16, True)
for form in F.GRAD_FORMS:
    F.test_gradient(form, int8.GRAD_WEIGHT)
    F.test_gradient(form, int8.GRAD_INPUT)
for form in F.PRODUCT_FORMS:
    F.test_product(form)
print("RESULT", json.dumps(int8.status()))
"""


def test_no_store_outside_its_range():
    r = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT}], capture_output=True, text=True, timeout=900, env=dict(os.environ, FMM_B200_DEBUG="1"))
    assert r.returncode == 0, r.stderr[-3000:]
    line = [ln for ln in r.stdout.splitlines() if ln.startswith("RESULT ")][-1]
    assert json.loads(line[len("RESULT "):]) == [0, 0]
