"""The product of 8-bit codes and its gradients against 64-bit products."""
import numpy as np
import pytest
import torch

import int8_oracle as O
from paper_2609_26077_b200 import int8

pytestmark = pytest.mark.gpu


def codes_of(rows, cols, seed, extreme=False):
    g = np.random.default_rng(seed)
    c = g.integers(-127, 128, (rows, cols), dtype=np.int64).astype(np.int8)
    if extreme and rows and cols:
        c[0], c[-1] = -128, 127
    return c


def scales_of(rows, seed, pow2=False):
    g = np.random.default_rng([seed, 1])
    s = np.exp(g.standard_normal(rows)).astype(np.float32) * np.float32(0.01)
    return np.exp2(np.round(np.log2(s))).astype(np.float32) if pow2 else s


def padded(c, extra=0):
    """On the device, rows a multiple of 16 bytes apart."""
    rows, cols = c.shape
    ld = -(-cols // 16) * 16 + extra
    buf = torch.full((rows, ld), 77, dtype=torch.int8, device="cuda")
    buf[:, :cols] = torch.from_numpy(c)
    return buf[:, :cols]


def check_matmul(M, N, K, dtype=torch.float32, bias=False, seed=0, extreme=True, extra=0, out=None):
    a, b, sa, sb = codes_of(M, K, seed, extreme), codes_of(N, K, seed + 1, extreme), scales_of(M, seed), scales_of(N, seed + 1)
    add = torch.randn(N, generator=torch.Generator().manual_seed(seed)).to(dtype) if bias else None
    c = int8.matmul(padded(a, extra), torch.from_numpy(sa).cuda(), padded(b, 2 * extra), torch.from_numpy(sb).cuda(),
                    bias=None if add is None else add.cuda(), dtype=dtype, out=out)
    acc = torch.from_numpy(a).cuda().double() @ torch.from_numpy(b).cuda().double().t()            # exact: whole numbers below 2^53
    want = (acc * torch.from_numpy(sa).cuda().double()[:, None] * torch.from_numpy(sb).cuda().double()).cpu().numpy()
    size = np.abs(want)
    if add is not None:
        want = want + O.host(add).astype(np.float64)
        size = size + np.abs(want)
    # the sum to fp32, two products, the bias: a rounding each; then the output's
    O.close(O.host(c), want, 4 * O.U32 * size + O.U[dtype] * np.abs(want) * 1.01 + O.TINY[dtype])
    return c


# as the library chooses by size (each kernel form by name: test_gpu_int8_forms.py); edges on each side
SHAPES = [(1, 1, 1), (1, 17, 31), (3, 100, 77), (5, 4737, 129), (8, 4800, 1000), (8, 15, 4100), (7, 2048, 2047), (9, 300, 300), (1, 8192, 8192), (1, 130, 64), (2, 257, 1000), (15, 513, 2048), (16, 128, 128), (17, 1024, 4096), (32, 640, 96), (33, 129, 257),
          (64, 4096, 512), (65, 200, 4095), (100, 3000, 200), (128, 128, 8192), (129, 127, 129), (300, 777, 640), (777, 2047, 2048), (1000, 33, 5000),
          (2048, 2048, 1024), (1500, 2500, 100), (2049, 1793, 384), (5000, 16, 256), (4097, 65, 64), (8192, 1, 130)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_matmul(M, N, K):
    check_matmul(M, N, K, bias=(M + N) % 2 == 0, seed=M + N)


def test_matmul_of_many_tiles_a_pair():
    """17 x 17 tiles of 256 x 256 among 74 pairs: both accumulators, every tile with the scales of its own columns."""
    check_matmul(4100, 4100, 2050, bias=True, seed=3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", [(1, 300, 512), (50, 70, 90), (200, 333, 1024), (2300, 2100, 256)])
def test_matmul_types(M, N, K, dtype):
    # (codes short of their limits keep the sums inside half precision's range)
    assert check_matmul(M, N, K, dtype, bias=True, seed=5, extreme=dtype is not torch.float16).dtype is dtype


def test_matmul_largest_sums():
    """Sums up to 2^31: every code at its limit, the longest K."""
    K = 131071
    for va, vb in ((-128, -128), (127, -128), (127, 127)):
        a = torch.full((3, 131072), va, dtype=torch.int8, device="cuda")[:, :K]
        b = torch.full((70, 131072), vb, dtype=torch.int8, device="cuda")[:, :K]
        c = int8.matmul(a, torch.ones(3, device="cuda"), b, torch.ones(70, device="cuda"), dtype=torch.float32)
        assert (c == float(np.float32(va * vb * K))).all()


def test_matmul_scales_far_apart():
    """A small scale times a large one: no overflow or underflow on the way to an ordinary result; NaN and infinite scales show."""
    a, b = codes_of(5, 64, 1), codes_of(6, 64, 2)
    sa = torch.tensor([1e-30, 1e30, 1.0, float("nan"), 2.0], device="cuda")
    sb = torch.tensor([1e30, 1e-30, 1.0, 1e30, 1e-30, float("nan")], device="cuda")
    c = int8.matmul(padded(a), sa, padded(b), sb, dtype=torch.float32).cpu().double()
    want = torch.from_numpy(a).double() @ torch.from_numpy(b).double().t() * sa.cpu().double()[:, None] * sb.cpu().double()
    inside = want.abs() < 3e38
    assert torch.isnan(c[3]).all() and torch.isnan(c[:, 5]).all()
    good = inside & ~torch.isnan(want) & (want.abs() > 1e-30)
    assert ((c - want)[good].abs() <= 4 * O.U32 * want[good].abs()).all() and good.sum() > 8
    assert torch.isinf(c[(want.abs() > 3.5e38)]).all()


def test_matmul_strided_output_and_operands():
    out = O.strided(torch.zeros(200, 333, device="cuda"), 5, 1)
    check_matmul(200, 333, 100, out=out, extra=48)
    assert torch.isnan(torch.as_strided(out, (199, 5), (338, 1), 1 + 333)).all()
    out = O.strided(torch.zeros(2100, 2001, dtype=torch.bfloat16, device="cuda"), 3, 1)
    check_matmul(2100, 2001, 200, torch.bfloat16, out=out, extra=16)
    assert torch.isnan(torch.as_strided(out, (2099, 3), (2004, 1), 1 + 2001).float()).all()


def test_matmul_empty():
    e = torch.empty(0, 64, dtype=torch.int8, device="cuda")
    b, sb = padded(codes_of(5, 64, 0)), torch.ones(5, device="cuda")
    assert int8.matmul(e, sb[:0], b, sb).shape == (0, 5)
    assert int8.matmul(b, sb, e, sb[:0]).shape == (5, 0)
    bias = torch.randn(5, device="cuda")
    none = torch.empty(3, 0, dtype=torch.int8, device="cuda")
    c = int8.matmul(none, sb[:3], torch.empty(5, 0, dtype=torch.int8, device="cuda"), sb, bias=bias, dtype=torch.float32)
    assert torch.equal(c, bias.expand(3, 5))


def test_matmul_refusals():
    b, s = padded(codes_of(8, 64, 0)), torch.ones(8, device="cuda")
    odd = torch.zeros(8, 65, dtype=torch.int8, device="cuda")
    for call in (lambda: int8.matmul(odd, s, odd, s), lambda: int8.matmul(b, s, b[:, :32], s), lambda: int8.matmul(b[:, 8:], s, b[:, 8:], s),
                 lambda: int8.matmul(b, s[:7], b, s), lambda: int8.matmul(b, s, b, s, bias=s.bfloat16()[:7])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: int8.matmul(b.float(), s, b, s), lambda: int8.matmul(b, s.half(), b, s), lambda: int8.matmul(b, s, b, s, dtype=torch.float64),
                 lambda: int8.matmul(b, s, b, s, bias=s)):
        with pytest.raises(TypeError):
            call()


# ------------------------------------------------------------------------------------------------ gradients
def restored(codes, scales, dtype):
    """Magnitudes of the restored values and how far each is off in `dtype`."""
    v = torch.from_numpy(O.values64(codes, scales)).cuda()
    return v, (v.to(torch.float32).to(dtype).double() - v).abs()


def check_grad(product, size, slip, got, contraction, out_type, old=None):
    # sums of exact products, a unit in the last place (2^-23) at most for each addition and never more than `contraction` of them;
    # slip: the restored operand's roundings
    want = product if old is None else product + old
    bound = contraction * 2 * O.U32 * size + slip + O.U[out_type] * want.abs() * 1.01 + O.TINY[out_type]
    if old is not None:
        bound = bound + 2 * O.U32 * (size + old.abs())
    O.close(O.host(got), want.cpu().numpy(), bound.cpu().numpy())


def check_grads(M, N, K, dtype=torch.bfloat16, out_type=torch.float32, pow2=True, seed=0, dy_extra=0, dy_offset=0):
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(M, N, generator=gen).to(dtype)
    x, sx, w, sw = codes_of(M, K, seed), scales_of(M, seed, pow2), codes_of(N, K, seed + 1), scales_of(N, seed + 1, pow2)
    d = dy.cuda().double()
    dyc = O.strided(dy.cuda(), dy_extra, dy_offset) if dy_extra or dy_offset else dy.cuda()
    dw = int8.grad_weight(dyc, padded(x), torch.from_numpy(sx).cuda(), dtype=out_type)
    v, off = restored(x, sx, dtype)
    check_grad(d.t() @ v, d.abs().t() @ v.abs(), d.abs().t() @ off, dw, M, out_type)
    dx = int8.grad_input(dyc, padded(w), torch.from_numpy(sw).cuda(), dtype=out_type)
    v, off = restored(w, sw, dtype)
    check_grad(d @ v, d.abs() @ v.abs(), d.abs() @ off, dx, N, out_type)
    return dw, dx


GRADS = [(1, 1, 1), (1, 64, 64), (3, 130, 70), (16, 64, 128), (33, 129, 257), (64, 64, 64), (100, 200, 300), (129, 128, 127), (257, 512, 1000), (1000, 65, 63),
         (1001, 2048, 2047), (2500, 300, 129), (300, 2304, 2200), (2048, 2048, 2048), (130, 4100, 1100)]


@pytest.mark.parametrize("M,N,K", GRADS)
def test_gradients(M, N, K):
    check_grads(M, N, K, seed=M + K)


@pytest.mark.parametrize("dtype,out_type,pow2", [(torch.bfloat16, torch.bfloat16, False), (torch.float16, torch.float16, False), (torch.float16, torch.float32, True),
                                                 (torch.bfloat16, torch.float32, False)])
@pytest.mark.parametrize("M,N,K", [(77, 200, 90), (700, 2100, 2200)])
def test_gradient_types(M, N, K, dtype, out_type, pow2):
    check_grads(M, N, K, dtype, out_type, pow2, seed=4)


@pytest.mark.parametrize("extra,offset", [(8, 0), (3, 0), (8, 1)])
def test_gradients_of_strided_dy(extra, offset):
    check_grads(130, 264, 200, seed=5, dy_extra=extra, dy_offset=offset)


@pytest.mark.parametrize("out_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(70, 130, 200), (500, 2200, 2100)])
def test_weight_gradient_accumulates(M, N, K, out_type):
    gen = torch.Generator().manual_seed(6)
    dy = torch.randn(M, N, generator=gen).bfloat16()
    x, sx = codes_of(M, K, 1), scales_of(M, 1, True)
    old = torch.randn(N, K, generator=gen).to(out_type)
    out = old.cuda()
    got = int8.grad_weight(dy.cuda(), padded(x), torch.from_numpy(sx).cuda(), out=out, accumulate=True)
    assert got is out
    d, (v, off) = dy.cuda().double(), restored(x, sx, torch.bfloat16)
    check_grad(d.t() @ v, d.abs().t() @ v.abs(), d.abs().t() @ off, got, M, out_type, old.cuda().double())


@pytest.mark.parametrize("out_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(70, 130, 200), (2100, 500, 2200)])
def test_input_gradient_accumulates(M, N, K, out_type):
    gen = torch.Generator().manual_seed(7)
    dy = torch.randn(M, N, generator=gen).bfloat16()
    w, sw = codes_of(N, K, 1), scales_of(N, 1, True)
    old = torch.randn(M, K, generator=gen).to(out_type)
    got = int8.grad_input(dy.cuda(), padded(w), torch.from_numpy(sw).cuda(), out=old.cuda(), accumulate=True)
    d, (v, off) = dy.cuda().double(), restored(w, sw, torch.bfloat16)
    check_grad(d @ v, d.abs() @ v.abs(), d.abs() @ off, got, N, out_type, old.cuda().double())


def test_gradients_of_nothing():
    dy = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    x = torch.empty(0, 40, dtype=torch.int8, device="cuda")
    assert not int8.grad_weight(dy, x, torch.empty(0, device="cuda")).any()
    old = torch.ones(24, 40, device="cuda")
    int8.grad_weight(dy, x, torch.empty(0, device="cuda"), out=old, accumulate=True)
    assert (old == 1).all()
    dy = torch.empty(8, 0, dtype=torch.bfloat16, device="cuda")
    dx = int8.grad_input(dy, x, torch.empty(0, device="cuda"))
    assert dx.shape == (8, 40) and not dx.any()


def test_gradient_refusals():
    dy, x, s = torch.zeros(8, 24, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 40, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda")
    for call in (lambda: int8.grad_weight(dy[:7], x, s), lambda: int8.grad_input(dy, x, s), lambda: int8.grad_weight(dy, x, s, accumulate=True),
                 lambda: int8.grad_weight(dy, x, s, out=torch.zeros(24, 41, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: int8.grad_weight(dy.float(), x, s), lambda: int8.grad_weight(dy, x, s, dtype=torch.float16)):
        with pytest.raises(TypeError):
            call()


def test_no_wait_gave_up():
    assert int8.status() == (0, 0)
