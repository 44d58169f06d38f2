"""Plain implementations of the 8-bit integer layer in numpy (not a test module): the quantizer step by step in IEEE single
precision, as include/fmm_int8.h defines it, and everything behind it in 64 bits."""
import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step, relative
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # smallest subnormal
TYPES = [torch.float32, torch.bfloat16, torch.float16]
U32 = U[torch.float32]


def blocks(x, block):
    rows, cols = x.shape
    block = block or max(cols, 1)
    per_row = -(-cols // block)
    padded = np.zeros((rows, per_row * block), x.dtype)
    padded[:, :cols] = x
    return padded.reshape(rows, per_row, block)


def quantize(x, block=0, pow2=False):
    """int8 codes and fp32 scales of a finite fp32 matrix."""
    x = np.asarray(x, np.float32)
    b = blocks(x, block)
    a = np.maximum(np.abs(b).max(2, initial=0.0), np.float32(1e-12)).astype(np.float32)
    scale = (a / np.float32(127)).astype(np.float32)
    if pow2:
        m, e = np.frexp(scale)
        scale = np.ldexp(np.float32(1), e - (m == 0.5)).astype(np.float32)
        inverse = (np.float32(1) / scale).astype(np.float32)
    else:
        inverse = (np.float32(127) / a).astype(np.float32)
    codes = np.rint((b * inverse[:, :, None]).astype(np.float32)).astype(np.int8)
    return codes.reshape(x.shape[0], -1)[:, :x.shape[1]], scale if block else scale.reshape(-1)


def values32(codes, scales, block=0):
    """code * scale rounded to fp32."""
    b = blocks(codes.astype(np.float32), block)
    v = (b * np.asarray(scales, np.float32).reshape(b.shape[0], b.shape[1])[:, :, None]).astype(np.float32)
    return v.reshape(codes.shape[0], -1)[:, :codes.shape[1]]


def values64(codes, scales, block=0):
    b = blocks(codes.astype(np.float64), block)
    v = b * np.asarray(scales, np.float64).reshape(b.shape[0], b.shape[1])[:, :, None]
    return v.reshape(codes.shape[0], -1)[:, :codes.shape[1]]


def rms_norm(x, gain, residual, eps):
    """hidden (fp32), rstd and normed rows (fp32) from fp32 inputs."""
    h = x if residual is None else (x + residual).astype(np.float32)
    rstd = (1.0 / np.sqrt((h.astype(np.float64) ** 2).sum(1) / h.shape[1] + eps)).astype(np.float32)
    return h, rstd, ((h * rstd[:, None]).astype(np.float32) * gain).astype(np.float32)


def rms_norm_backward(dy, h, rstd, gain, dresidual):
    """dx, dgain and the magnitudes that their rounding errors are measured by, in 64 bits."""
    n = max(h.shape[1], 1)
    xhat = h * rstd[:, None]
    g = dy * gain
    c = (g * xhat).sum(1, keepdims=True) / n
    dx = rstd[:, None] * (g - xhat * c)
    size = rstd[:, None] * (np.abs(g) + np.abs(xhat) * (np.abs(g * xhat).sum(1, keepdims=True) / n))
    if dresidual is not None:
        dx, size = dx + dresidual, size + np.abs(dresidual)
    return dx, size, (dy * xhat).sum(0), np.abs(dy * xhat).sum(0)


# ---------------------------------------------------------------- tensors
def host(t):
    """A tensor's numbers, exactly, as fp32 (int8 as int8)."""
    t = t.detach().cpu()
    return t.numpy() if t.dtype == torch.int8 else t.float().numpy()


def strided(t, extra, offset=0):
    """The same matrix with `extra` elements of poison behind every row, `offset` elements behind an aligned address."""
    rows, cols = t.shape
    poison = 85 if t.dtype == torch.int8 else float("nan")
    buf = torch.full((rows * (cols + extra) + offset + 1,), poison, dtype=t.dtype, device=t.device)
    view = buf[offset:offset + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
    view.copy_(t)
    return view


def close(got, want, bound):
    """Every element within its bound; the worst ratio in the message."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    off = np.abs(got - want)
    bad = ~(off <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} elements off, at worst {np.max(off / np.maximum(bound, 1e-300)):.3g} times the bound"
