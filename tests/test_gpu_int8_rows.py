"""Quantization, restoring, the norm with 8-bit output and its gradients against the oracle: codes and scales bit for bit."""
import numpy as np
import pytest
import torch

import int8_oracle as O
from paper_2609_26077_b200 import fmm, int8

pytestmark = pytest.mark.gpu

# one column, odd ones, around 8 (a thread's columns), 32 and 128 (blocks), 512, 1024, 8192 (kernels), 16384 and behind (long rows)
COLS = [1, 7, 31, 33, 127, 130, 512, 520, 1000, 1024, 1032, 2048, 2056, 4095, 5120, 8192, 8200, 16384]
LONG = [16392, 40001]


def rows_of(rows, cols, dtype, seed, spread=1.5):
    """Rows with a lognormal factor per channel and one per row, one row of zeros and one of tiny numbers."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(cols, generator=g)) * torch.exp(torch.randn(rows, 1, generator=g))
    if rows > 2:
        x[1] = 0
        x[2] *= 1e-6
    return x.to(dtype)


def check_quantized(codes, scales, want, what):
    wc, ws = want
    assert np.array_equal(O.host(scales), ws), f"{what}: scales"
    assert np.array_equal(O.host(codes), wc), f"{what}: codes"


@pytest.mark.parametrize("dtype", O.TYPES)
@pytest.mark.parametrize("block,pow2", [(0, False), (0, True), (32, False), (32, True), (128, False), (128, True)])
def test_quantize_is_bit_exact(dtype, block, pow2):
    for i, cols in enumerate(COLS + LONG):
        rows = (1, 5, 3)[i % 3]
        x = rows_of(rows, cols, dtype, i)
        codes, scales = int8.quantize(x.cuda(), block=block, pow2=pow2)
        check_quantized(codes, scales, O.quantize(O.host(x), block, pow2), f"{rows} x {cols}")
        # restored: the fp32 product, rounded once
        for out in O.TYPES:
            back = int8.dequantize(codes, scales, block=block, dtype=out)
            want = torch.from_numpy(O.values32(O.host(codes), O.host(scales), block)).to(out)
            assert torch.equal(back.cpu(), want), (rows, cols, out)


def test_quantize_many_rows():
    x = rows_of(9001, 96, torch.bfloat16, 3)
    for block in (0, 32):
        codes, scales = int8.quantize(x.cuda(), block=block)
        check_quantized(codes, scales, O.quantize(O.host(x), block), f"block {block}")
        assert torch.equal(int8.dequantize(codes, scales, block, torch.float32).cpu(), torch.from_numpy(O.values32(O.host(codes), O.host(scales), block)))


def test_quantize_ties_and_limits():
    # multiples of half a step: ties go to the even code; the largest finite numbers; powers of two and their neighbours
    base = torch.arange(-127, 127.5, 0.5).repeat(2, 1)
    base[1] *= 2.0 ** 119
    codes, scales = int8.quantize(base.cuda())
    check_quantized(codes, scales, O.quantize(base.numpy()), "ties")
    top = torch.tensor([[3.4028234e38, -1e38, 1.0], [127.0, 1.0, 0.5], [127.00001, 63.5, -0.25], [126.99999, 64.5, 2.0 ** -149]])
    for pow2 in (False, True):
        codes, scales = int8.quantize(top.cuda(), pow2=pow2)
        check_quantized(codes, scales, O.quantize(top.numpy(), pow2=pow2), f"pow2 {pow2}")


def test_infinities_and_nan_stay_in_their_block():
    x = torch.ones(4, 300)
    x[0, 5], x[1, 290], x[2, 0] = float("nan"), float("inf"), float("-inf")
    for block in (0, 32, 128):
        for pow2 in (False, True):
            codes, scales = int8.quantize(x.cuda(), block=block, pow2=pow2)
            v = int8.dequantize(codes, scales, block=block, dtype=torch.float32).cpu()
            width = block or 300
            for r, c in ((0, 5), (1, 290), (2, 0)):
                lo = c // width * width
                assert torch.isnan(v[r, lo:lo + width]).all()
                assert torch.isfinite(v[r, :lo]).all() and torch.isfinite(v[r, lo + width:]).all()
            assert torch.isfinite(v[3]).all()


@pytest.mark.parametrize("extra,offset", [(8, 0), (3, 1), (5, 2)])
def test_strides_and_alignment(extra, offset):
    """Rows any distance apart at any address: the same results, and nothing behind a row is touched."""
    x = rows_of(6, 515, torch.float16, 4)
    xs = O.strided(x.cuda(), extra, offset)
    for block in (0, 32):
        want = O.quantize(O.host(x), block)
        codes = O.strided(torch.zeros(6, 515, dtype=torch.int8, device="cuda"), extra, offset)
        scales = torch.empty(int8._scale_shape(6, 515, block), device="cuda")
        int8.quantize(xs, block=block, out=(codes, scales))
        check_quantized(codes, scales, want, "strided")
        gap = torch.as_strided(codes, (5, extra), (515 + extra, 1), codes.storage_offset() + 515)
        assert (gap == 85).all()
        out = O.strided(torch.zeros(6, 515, dtype=torch.float16, device="cuda"), extra, offset)
        int8.dequantize(codes, scales, block=block, out=out)
        assert torch.equal(out.cpu(), torch.from_numpy(O.values32(*want, block)).half())
        assert torch.isnan(torch.as_strided(out, (5, extra), (515 + extra, 1), out.storage_offset() + 515)).all()


def test_empty_matrices():
    for rows, cols in ((0, 64), (3, 0), (0, 0)):
        x = torch.empty(rows, cols, device="cuda")
        codes, scales = int8.quantize(x)
        assert codes.shape == (rows, cols) and scales.shape == (rows,)
        assert int8.dequantize(codes, scales).shape == (rows, cols)
    dx, dgain = int8.rms_norm_backward(torch.empty(0, 64, device="cuda"), torch.empty(0, 64, dtype=torch.int8, device="cuda"),
                                       torch.empty(0, 2, device="cuda"), torch.empty(0, device="cuda"), torch.ones(64, device="cuda"), block=32)
    assert dx.shape == (0, 64) and not dgain.any()


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("dtype", O.TYPES)
def test_rows_without_columns_touch_nothing(dtype, pow2):
    """Views of no columns in aligned buffers whose rows are 64 and 512 elements apart: the scales of nothing, the buffers as they were."""
    for ld in (64, 512):
        x, codes = torch.full((5, ld), float("nan"), dtype=dtype, device="cuda"), torch.full((5, ld), 77, dtype=torch.int8, device="cuda")
        scales = torch.full((7,), -1.0, device="cuda")
        want = O.quantize(np.zeros((5, 1), np.float32), 0, pow2)[1]          # a row of zeros has the same scale
        got = int8.quantize(x[:, :0], pow2=pow2, out=(codes[:, :0], scales[:5]))
        assert got[0].shape == (5, 0)
        assert np.array_equal(O.host(scales[:5]), want) and (scales[5:] == -1).all()
        assert (codes == 77).all() and torch.isnan(x).all()
        # by addresses, as a C caller has them: present, and absent
        for at_x, at_codes in ((x.data_ptr(), codes.data_ptr()), (0, 0)):
            a = int8._quantize_args(int8._TYPES[dtype], 0, int8.POW2 if pow2 else int8.AMAX_DIV_127, 5, 0, at_x, 0, at_codes, 0, scales.data_ptr())
            scales.fill_(-1.0)
            assert int8.lib().fmm_int8_quantize(a, torch.cuda.current_stream().cuda_stream) == 0
            assert np.array_equal(O.host(scales[:5]), want) and (scales[5:] == -1).all()
            assert (codes == 77).all()


# ------------------------------------------------------------------------------------------------ norm
def norm_case(rows, cols, dtype, seed, residual=True):
    g = torch.Generator().manual_seed(1000 + seed)
    x = rows_of(rows, cols, dtype, seed)
    r = rows_of(rows, cols, dtype, seed + 50) if residual else None
    gain = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype)
    return x, r, gain


def check_norm(x, r, gain, n, pow2, block, eps=1e-6):
    h, rstd, y = O.rms_norm(O.host(x), O.host(gain), None if r is None else O.host(r), eps)
    assert np.array_equal(O.host(n.rstd), rstd)
    check_quantized(n.codes, n.scales, O.quantize(y, 0, pow2), "norm")
    if r is not None:
        assert torch.equal(n.hidden.cpu(), torch.from_numpy(h).to(x.dtype))
    if block:
        check_quantized(n.checkpoint, n.checkpoint_scales, O.quantize(h, block), "checkpoint")


@pytest.mark.parametrize("dtype", O.TYPES)
@pytest.mark.parametrize("residual,pow2,block", [(True, False, 0), (True, True, 128), (False, False, 32), (True, False, 32)])
def test_norm_is_bit_exact(dtype, residual, pow2, block):
    for i, cols in enumerate(COLS + LONG):
        rows = (1, 4, 7)[i % 3]
        x, r, gain = norm_case(rows, cols, dtype, i, residual)
        cuda = [None if t is None else t.cuda() for t in (x, r, gain)]
        n = int8.rms_norm(cuda[0], cuda[2], residual=cuda[1], pow2=pow2, checkpoint=block)
        check_norm(x, r, gain, n, pow2, block)
        if not residual:
            assert n.hidden is cuda[0]


@pytest.mark.parametrize("cols", [300, 16500])
@pytest.mark.parametrize("into", ["x", "residual"])
def test_norm_in_place(cols, into):
    x, r, gain = norm_case(5, cols, torch.bfloat16, 7)
    a, b = x.cuda(), r.cuda()
    n = int8.rms_norm(a, gain.cuda(), residual=b, checkpoint=32, hidden=a if into == "x" else b)
    check_norm(x, r, gain, n, False, 32)
    assert n.hidden is (a if into == "x" else b)
    assert torch.equal((b if into == "x" else a).cpu(), r if into == "x" else x)


def test_norm_strided_and_row_of_zeros():
    x, r, gain = norm_case(5, 515, torch.float32, 9)
    x[3] = 0
    r[3] = 0
    hidden = O.strided(torch.zeros(5, 515, device="cuda"), 3, 1)
    n = int8.rms_norm(O.strided(x.cuda(), 5, 3), gain.cuda(), residual=O.strided(r.cuda(), 1, 1), hidden=hidden)
    check_norm(x, r, gain, n, False, 0)
    assert torch.isnan(torch.as_strided(hidden, (4, 3), (518, 1), 1 + 515)).all()
    assert n.rstd[3].item() == pytest.approx(1e3, rel=1e-6) and not n.codes[3].any()


def test_norm_with_nan_and_infinite_rows():
    x, _, gain = norm_case(4, 700, torch.bfloat16, 11, residual=False)
    x[0, 3], x[2, 699] = float("nan"), float("inf")
    n = int8.rms_norm(x.cuda(), gain.cuda(), checkpoint=128)
    v = int8.dequantize(n.codes, n.scales).cpu()
    k = int8.dequantize(n.checkpoint, n.checkpoint_scales, block=128).cpu()
    assert torch.isnan(v[0]).all() and torch.isnan(v[2]).any() and torch.isfinite(v[[1, 3]]).all()
    assert torch.isnan(k[0, :128]).all() and torch.isfinite(k[0, 128:]).all() and torch.isnan(k[2, 640:]).all()


# ------------------------------------------------------------------------------------------------ the norm's gradients
def back_case(rows, cols, dtype, block, seed, residual=True):
    g = torch.Generator().manual_seed(2000 + seed)
    h = rows_of(rows, cols, torch.float32, seed)
    codes, scales = O.quantize(h.numpy(), block)
    rstd = (1 / np.sqrt((h.numpy().astype(np.float64) ** 2).mean(1) + 1e-6)).astype(np.float32)
    dy = torch.randn(rows, cols, generator=g).to(dtype)
    gain = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype)
    dres = torch.randn(rows, cols, generator=g).to(dtype) if residual else None
    return codes, scales, rstd, dy, gain, dres


def check_back(case, dx, dgain, block):
    codes, scales, rstd, dy, gain, dres = case
    want, size, wgain, gsize = O.rms_norm_backward(O.host(dy).astype(np.float64), O.values64(codes, scales, block), rstd.astype(np.float64),
                                                   O.host(gain).astype(np.float64), None if dres is None else O.host(dres).astype(np.float64))
    rows, cols = codes.shape
    # dx: each number passes fewer than 16 roundings of its own; the row's sum fewer than 8 * (groups of 8 a thread) + 20.  Rounded to
    # the type once, half a step
    sums = 8 * -(-cols // 8192) + 8 * 4 + 20
    O.close(O.host(dx), want, (sums + 16) * O.U32 * size + O.U[dy.dtype] * np.abs(want) * 1.01 + O.TINY[dy.dtype])
    # dgain: products with three roundings, at most rows + 64 additions
    O.close(O.host(dgain), wgain, (rows + 68) * O.U32 * gsize + 1e-37)


@pytest.mark.parametrize("dtype", O.TYPES)
@pytest.mark.parametrize("block,residual", [(32, True), (128, False), (0, True)])
def test_norm_backward(dtype, block, residual):
    for i, cols in enumerate(COLS + LONG):
        rows = (1, 6, 19)[i % 3]
        case = back_case(rows, cols, dtype, block, i, residual)
        codes, scales, rstd, dy, gain, dres = [None if t is None else torch.as_tensor(t).cuda() for t in case]
        dx, dgain = int8.rms_norm_backward(dy, codes, scales, rstd, gain, block=block, dresidual=dres)
        check_back(case, dx, dgain, block)


def test_norm_backward_many_rows_is_deterministic():
    case = back_case(5000, 264, torch.bfloat16, 32, 1)
    args = [torch.as_tensor(t).cuda() for t in case]
    codes, scales, rstd, dy, gain, dres = args
    first = int8.rms_norm_backward(dy, codes, scales, rstd, gain, block=32, dresidual=dres)
    check_back(case, *first, 32)
    again = int8.rms_norm_backward(dy, codes, scales, rstd, gain, block=32, dresidual=dres)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("cols", [520, 17000])
@pytest.mark.parametrize("into", ["dy", "dresidual"])
def test_norm_backward_in_place_and_strided(cols, into):
    case = back_case(37, cols, torch.float16, 128, 3)
    codes, scales, rstd, dy, gain, dres = [torch.as_tensor(t).cuda() for t in case]
    dy, dres, codes = O.strided(dy, 3, 1), O.strided(dres, 8, 0), O.strided(codes, 5, 3)
    out = dy if into == "dy" else dres
    dx, dgain = int8.rms_norm_backward(dy, codes, scales, rstd, gain, dresidual=dres, dx=out)
    assert dx is out
    check_back(case, dx, dgain, 128)


def test_norm_backward_against_differences():
    """The gradient at the checkpoint's own values, where rstd is their own: central differences of the 64-bit norm."""
    rows, cols, block = 3, 48, 32
    codes, scales, _, dy, gain, _ = back_case(rows, cols, torch.float32, block, 5, residual=False)
    h = O.values64(codes, scales, block)
    eps = 1e-6
    rstd = (1 / np.sqrt((h ** 2).mean(1) + eps)).astype(np.float32)
    dx, dgain = int8.rms_norm_backward(*[torch.as_tensor(t).cuda() for t in (dy, codes, scales, rstd, gain)], block=block)
    g, d = O.host(gain).astype(np.float64), O.host(dy).astype(np.float64)

    def loss(h, g):
        return (d * h / np.sqrt((h ** 2).mean(1, keepdims=True) + eps) * g).sum(1)
    got = O.host(dx)
    for c in range(cols):
        step = 1e-4 * np.sqrt((h ** 2).mean(1) + eps)
        up, down = h.copy(), h.copy()
        up[:, c] += step
        down[:, c] -= step
        slope = (loss(up, g) - loss(down, g)) / (2 * step)
        # the differences' own error is of the order of (step / rms)^2 = 1e-8 of the gradient's size
        assert np.all(np.abs(got[:, c] - slope) <= 1e-5 * np.abs(got).max(1))
        gu, gd = g.copy(), g.copy()
        gu[c] += 1e-4
        gd[c] -= 1e-4
        assert O.host(dgain)[c] == pytest.approx(((loss(h, gu) - loss(h, gd)) / 2e-4).sum(), rel=1e-5, abs=1e-5)


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    codes, scales = int8.quantize(x)
    for call in (lambda: int8.quantize(x, block=64), lambda: int8.quantize(x.t()), lambda: int8.quantize(x[0]),
                 lambda: int8.quantize(x.expand(4, 64)[:1].expand(4, 64)), lambda: int8.dequantize(codes, scales[:3]),
                 lambda: int8.rms_norm(x, torch.ones(63, device="cuda")), lambda: int8.rms_norm(x, x[0], hidden=x),
                 lambda: int8.rms_norm(x, x[0], residual=x[:3])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: int8.quantize(codes), lambda: int8.quantize(x.double()), lambda: int8.dequantize(codes, scales.cpu()),
                 lambda: int8.rms_norm(x, x[0].half()), lambda: int8.rms_norm_backward(x, codes, scales, scales, x[0].half(), block=0)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(fmm.FmmError):
        int8.rms_norm(x, x[0], eps=-1.0)


def test_refusals_of_numbers_and_streams():
    """Arguments that are no tensors: the errors that the binding states, not those of its packing."""
    x = torch.zeros(4, 64, device="cuda")
    codes, scales = int8.quantize(x)
    for call in (lambda: int8.rms_norm(x, x[0], checkpoint=None), lambda: int8.rms_norm(x, x[0], checkpoint=32.0), lambda: int8.rms_norm(x, x[0], eps=None),
                 lambda: int8.rms_norm(x, x[0], eps="small"), lambda: int8.quantize(x, block=None), lambda: int8.quantize(x, block=32.0),
                 lambda: int8.dequantize(codes, scales, block="32"), lambda: int8.rms_norm_backward(x, codes, scales, scales, x[0], block=None),
                 lambda: int8.quantize(x, stream=0), lambda: int8.dequantize(codes, scales, dtype=None), lambda: int8.matmul(codes, scales, codes, scales, stream="s")):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: int8.rms_norm(x, x[0], checkpoint=64), lambda: int8.rms_norm_backward(x, codes, scales, scales, x[0], block=-1)):
        with pytest.raises(ValueError):
            call()
    for eps in (float("nan"), float("inf"), -1):
        with pytest.raises(fmm.FmmError):
            int8.rms_norm(x, x[0], eps=eps)
    n = int8.rms_norm(x, x[0], eps=np.float32(1e-6), checkpoint=np.int64(32))
    assert n.checkpoint_scales.shape == (4, 2)


def test_nothing_is_recorded_for_autograd():
    w = torch.nn.Parameter(torch.randn(4, 64, device="cuda"))
    codes, scales = int8.quantize(w)
    assert not scales.requires_grad and not int8.dequantize(codes, scales).requires_grad
