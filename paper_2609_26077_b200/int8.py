"""The 8-bit integer layer of libfmm_b200.so: ctypes binding of include/fmm_int8.h (argument checks and marshalling only;
every step runs in the CUDA kernels).

A forward and backward pass of one layer, everything that is kept for the backward pass in 8 bits:

    w, ws = int8.quantize(weight)                                   # (N, K): one scale per output channel
    n = int8.rms_norm(x, gain, residual=r, checkpoint=128)          # hidden rows, their 8-bit norm, a checkpoint
    z = int8.matmul(n.codes, n.scales, w, ws)                       # (M, N)
    ...
    dw = int8.grad_weight(dz, n.codes, n.scales)                    # (N, K)
    dy = int8.grad_input(dz, w, ws)                                 # (M, K)
    dx, dgain = int8.rms_norm_backward(dy, n.checkpoint, n.checkpoint_scales, n.rstd, gain, block=128, dresidual=dh)

Matrices are 2-D CUDA tensors whose columns are contiguous (rows may lie any distance apart); scales and gains are
contiguous.  All tensors of a call are on one device, on whose current stream the work is enqueued, or on `stream`; nothing
is synchronised, and calls may be captured into CUDA graphs.  Outputs are allocated unless they are given; codes get rows
that are a multiple of 16 bytes apart, as `matmul` wants them.  Unsuitable tensors raise TypeError (types, devices) or
ValueError (shapes, strides), anything that the library refuses raises fmm.FmmError.
"""
from __future__ import annotations

import collections
import contextlib
import ctypes as C

import torch

from . import fmm

AMAX_DIV_127, POW2 = 0, 1
F32, BF16, F16 = 0, 1, 2
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

EXPORTS = ["fmm_int8_quantize", "fmm_int8_dequantize", "fmm_int8_rms_norm", "fmm_int8_rms_norm_backward_workspace_bytes",
           "fmm_int8_rms_norm_backward", "fmm_int8_matmul", "fmm_int8_grad_workspace_bytes", "fmm_int8_grad_weight",
           "fmm_int8_grad_input", "fmm_int8_status", "fmm_int8_status_clear"]


class RmsNormArgs(C.Structure):
    """fmm_int8_rms_norm_t"""
    _fields_ = [("type", C.c_int), ("scale_mode", C.c_int), ("checkpoint_block", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64),
                ("eps", C.c_double), ("x", C.c_void_p), ("ldx", C.c_int64), ("residual", C.c_void_p), ("ldr", C.c_int64),
                ("gain", C.c_void_p), ("hidden", C.c_void_p), ("ldh", C.c_int64), ("codes", C.c_void_p), ("ldc", C.c_int64),
                ("scales", C.c_void_p), ("rstd", C.c_void_p), ("checkpoint", C.c_void_p), ("ldk", C.c_int64),
                ("checkpoint_scales", C.c_void_p)]


class RmsNormBackwardArgs(C.Structure):
    """fmm_int8_rms_norm_backward_t"""
    _fields_ = [("type", C.c_int), ("block", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64), ("dy", C.c_void_p), ("ldy", C.c_int64),
                ("checkpoint", C.c_void_p), ("ldk", C.c_int64), ("checkpoint_scales", C.c_void_p), ("rstd", C.c_void_p),
                ("gain", C.c_void_p), ("dresidual", C.c_void_p), ("ldr", C.c_int64), ("dx", C.c_void_p), ("ldx", C.c_int64),
                ("dgain", C.c_void_p)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = fmm.lib()
        ptr, i64, i32, size = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
        L.fmm_int8_quantize.argtypes = [ptr, i32, i64, i64, i64, i32, i32, ptr, i64, ptr, ptr]
        L.fmm_int8_dequantize.argtypes = [ptr, i64, ptr, i64, i64, i32, ptr, i32, i64, ptr]
        L.fmm_int8_rms_norm.argtypes = [ptr, ptr]
        L.fmm_int8_rms_norm_backward_workspace_bytes.argtypes = [i64, i64, ptr]
        L.fmm_int8_rms_norm_backward.argtypes = [ptr, ptr, size, ptr]
        L.fmm_int8_matmul.argtypes = [ptr, i64, ptr, ptr, i64, ptr, ptr, i64, i64, i64, ptr, i32, i64, ptr]
        L.fmm_int8_grad_workspace_bytes.argtypes = [i64, i64, i64, i64, i32, ptr]
        L.fmm_int8_grad_weight.argtypes = [ptr, i32, i64, ptr, i64, ptr, i64, i64, i64, ptr, i32, i64, i32, ptr, size, ptr]
        L.fmm_int8_grad_input.argtypes = [ptr, i32, i64, ptr, i64, ptr, i64, i64, i64, ptr, i32, i64, ptr, size, ptr]
        L.fmm_int8_status.argtypes = [ptr]
        _lib = L
    return _lib


# ------------------------------------------------------------------------------------------------ checks
def _matrix(t, name, dtype, shape=None):
    """A 2-D CUDA tensor with contiguous columns; its row distance."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: a CUDA tensor is needed")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype} is needed, not {t.dtype}")
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, {'two dimensions are' if shape is None else f'{shape} is'} needed")
    rows, cols = t.shape
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{name}: columns are not contiguous")
    if rows > 1:
        if ld < cols:
            raise ValueError(f"{name}: rows overlap or run backwards")
        return ld
    return max(ld, cols) if cols > 1 else max(cols, 1)


def _vector(t, name, dtype, shape):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: a CUDA tensor is needed")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype} is needed, not {t.dtype}")
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor of shape {shape} is needed, not {tuple(t.shape)}")


def _float_type(dtype, name):
    if dtype not in _TYPES:
        raise TypeError(f"{name}: float32, bfloat16 or float16 is needed, not {dtype}")
    return _TYPES[dtype]


def _block(block, name="block"):
    if block not in (0, 32, 128):
        raise ValueError(f"{name}: 0, 32 or 128 is needed, not {block!r}")
    return block


def _scale_shape(rows, cols, block):
    return (rows, -(-cols // block)) if block else (rows,)


def _same_device(first, *tensors):
    for t in tensors:
        if t is not None and t.device != first.device:
            raise TypeError(f"tensors on {first.device} and {t.device} in one call")


_here = contextlib.nullcontext()


def _on(t, stream):
    """The context in which a call on t's device and on `stream` allocates and launches."""
    if stream is not None:
        if stream.device != t.device:
            raise TypeError(f"a stream of {stream.device} for tensors on {t.device}")
        return torch.cuda.stream(stream)
    return _here if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)


def _new_codes(rows, cols, device):
    """Codes whose rows are a multiple of 16 bytes apart."""
    if cols % 16 == 0:
        return torch.empty((rows, cols), dtype=torch.int8, device=device)
    return torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=device)[:, :cols]


def _new(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


def _call(status, what):
    if status:
        fmm._check(status, what)


# ------------------------------------------------------------------------------------------------ operators
def quantize(x, block=0, pow2=False, out=None, stream=None):
    """Codes and scales of x (rows x cols): one scale per row, or per block of 32 or 128 columns of a row; with pow2 each is
    a power of two.  out: (codes, scales) to write to."""
    kind = _float_type(x.dtype, "x")
    ldx = _matrix(x, "x", x.dtype)
    rows, cols = x.shape
    shape = _scale_shape(rows, cols, _block(block))
    with _on(x, stream):
        codes, scales = out if out is not None else (_new_codes(rows, cols, x.device), _new(shape, torch.float32, x.device))
        ldc = _matrix(codes, "codes", torch.int8, (rows, cols))
        _vector(scales, "scales", torch.float32, shape)
        _same_device(x, codes, scales)
        _call(lib().fmm_int8_quantize(x.data_ptr(), kind, ldx, rows, cols, block, POW2 if pow2 else AMAX_DIV_127, codes.data_ptr(), ldc,
                                      scales.data_ptr(), fmm._stream_ptr(None)), "fmm_int8_quantize")
    return codes, scales


def dequantize(codes, scales, block=0, dtype=torch.bfloat16, out=None, stream=None):
    """The values that codes stand for, code * scale, in `dtype` (or out's type)."""
    ldc = _matrix(codes, "codes", torch.int8)
    rows, cols = codes.shape
    _vector(scales, "scales", torch.float32, _scale_shape(rows, cols, _block(block)))
    with _on(codes, stream):
        if out is None:
            kind, out = _float_type(dtype, "dtype"), _new((rows, cols), dtype, codes.device)
        else:
            kind = _float_type(out.dtype, "out")
        ldx = _matrix(out, "out", out.dtype, (rows, cols))
        _same_device(codes, scales, out)
        _call(lib().fmm_int8_dequantize(codes.data_ptr(), ldc, scales.data_ptr(), rows, cols, block, out.data_ptr(), kind, ldx,
                                        fmm._stream_ptr(None)), "fmm_int8_dequantize")
    return out


Norm = collections.namedtuple("Norm", "hidden codes scales rstd checkpoint checkpoint_scales")


def rms_norm(x, gain, residual=None, eps=1e-6, pow2=False, checkpoint=0, hidden=None, stream=None):
    """Norm(hidden, codes, scales, rstd, checkpoint, checkpoint_scales) of h = x + residual:

        hidden                         h in x's type (x itself without a residual); written to `hidden` where that is given,
                                       which may be x or residual
        codes, scales                  8-bit form, a scale per row, of h / rms(h) * gain
        rstd                           1 / rms(h) per row
        checkpoint, checkpoint_scales  8-bit form of h in blocks of `checkpoint` (32 or 128) columns; None with 0
    """
    kind = _float_type(x.dtype, "x")
    a = RmsNormArgs(kind, POW2 if pow2 else AMAX_DIV_127, _block(checkpoint, "checkpoint"))
    a.ldx = _matrix(x, "x", x.dtype)
    rows, cols = x.shape
    _vector(gain, "gain", x.dtype, (cols,))
    with _on(x, stream):
        if residual is not None:
            a.ldr = _matrix(residual, "residual", x.dtype, (rows, cols))
            if hidden is None:
                hidden = _new((rows, cols), x.dtype, x.device)
            a.ldh = _matrix(hidden, "hidden", x.dtype, (rows, cols))
            a.residual, a.hidden = residual.data_ptr(), hidden.data_ptr()
        elif hidden is not None:
            raise ValueError("hidden: written with a residual only")
        codes, scales, rstd = _new_codes(rows, cols, x.device), _new((rows,), torch.float32, x.device), _new((rows,), torch.float32, x.device)
        kept = kept_scales = None
        if checkpoint:
            kept, kept_scales = _new_codes(rows, cols, x.device), _new(_scale_shape(rows, cols, checkpoint), torch.float32, x.device)
            a.checkpoint, a.ldk, a.checkpoint_scales = kept.data_ptr(), kept.stride(0), kept_scales.data_ptr()
        _same_device(x, gain, residual, hidden)
        a.rows, a.cols, a.eps, a.x, a.gain = rows, cols, eps, x.data_ptr(), gain.data_ptr()
        a.codes, a.ldc, a.scales, a.rstd = codes.data_ptr(), codes.stride(0), scales.data_ptr(), rstd.data_ptr()
        _call(lib().fmm_int8_rms_norm(C.byref(a), fmm._stream_ptr(None)), "fmm_int8_rms_norm")
    return Norm(x if residual is None else hidden, codes, scales, rstd, kept, kept_scales)


def rms_norm_backward(dy, checkpoint, checkpoint_scales, rstd, gain, block=128, dresidual=None, dx=None, stream=None):
    """(dx, dgain) of the norm, from the checkpoint of its hidden rows and their rstd.  dx, the gradient of x and of residual,
    includes dresidual, the gradient that reaches the hidden rows elsewhere; it may be dy or dresidual.  dgain is float32."""
    kind = _float_type(dy.dtype, "dy")
    a = RmsNormBackwardArgs(kind, _block(block))
    a.ldy = _matrix(dy, "dy", dy.dtype)
    rows, cols = dy.shape
    a.ldk = _matrix(checkpoint, "checkpoint", torch.int8, (rows, cols))
    _vector(checkpoint_scales, "checkpoint_scales", torch.float32, _scale_shape(rows, cols, block))
    _vector(rstd, "rstd", torch.float32, (rows,))
    _vector(gain, "gain", dy.dtype, (cols,))
    with _on(dy, stream):
        if dresidual is not None:
            a.ldr = _matrix(dresidual, "dresidual", dy.dtype, (rows, cols))
            a.dresidual = dresidual.data_ptr()
        if dx is None:
            dx = _new((rows, cols), dy.dtype, dy.device)
        a.ldx = _matrix(dx, "dx", dy.dtype, (rows, cols))
        _same_device(dy, checkpoint, checkpoint_scales, rstd, gain, dresidual, dx)
        dgain = _new((cols,), torch.float32, dy.device)
        need = C.c_size_t()
        _call(lib().fmm_int8_rms_norm_backward_workspace_bytes(rows, cols, C.byref(need)), "fmm_int8_rms_norm_backward_workspace_bytes")
        workspace = _new((need.value,), torch.uint8, dy.device)
        a.rows, a.cols, a.dy, a.checkpoint, a.checkpoint_scales = rows, cols, dy.data_ptr(), checkpoint.data_ptr(), checkpoint_scales.data_ptr()
        a.rstd, a.gain, a.dx, a.dgain = rstd.data_ptr(), gain.data_ptr(), dx.data_ptr(), dgain.data_ptr()
        _call(lib().fmm_int8_rms_norm_backward(C.byref(a), workspace.data_ptr(), need.value, fmm._stream_ptr(None)), "fmm_int8_rms_norm_backward")
    return dx, dgain


def matmul(a, a_scales, b, b_scales, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """a (M x K codes, a scale per row) times the transpose of b (N x K codes, a scale per row), plus bias (N): M x N in
    `dtype` (or out's type).  The rows of a and b start on 16-byte boundaries; K is at most 131071."""
    lda = _matrix(a, "a", torch.int8)
    M, K = a.shape
    ldb = _matrix(b, "b", torch.int8)
    N = b.shape[0]
    if b.shape[1] != K:
        raise ValueError(f"a and b have {K} and {b.shape[1]} columns")
    # a single row need not be any distance from the next
    lda, ldb = lda if M > 1 else (K + 15) // 16 * 16, ldb if N > 1 else (K + 15) // 16 * 16
    if K and (lda % 16 or ldb % 16 or (M and a.data_ptr() % 16) or (N and b.data_ptr() % 16)):
        raise ValueError("a and b: rows have to start on 16-byte boundaries (as those of quantize and rms_norm do)")
    _vector(a_scales, "a_scales", torch.float32, (M,))
    _vector(b_scales, "b_scales", torch.float32, (N,))
    with _on(a, stream):
        if out is None:
            kind, out = _float_type(dtype, "dtype"), _new((M, N), dtype, a.device)
        else:
            kind = _float_type(out.dtype, "out")
        ldc = _matrix(out, "out", out.dtype, (M, N))
        if bias is not None:
            _vector(bias, "bias", out.dtype, (N,))
        _same_device(a, a_scales, b, b_scales, bias, out)
        _call(lib().fmm_int8_matmul(a.data_ptr(), lda, a_scales.data_ptr(), b.data_ptr(), ldb, b_scales.data_ptr(),
                                    None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), kind, ldc, fmm._stream_ptr(None)),
              "fmm_int8_matmul")
    return out


def _grad(what, dy, codes, scales, shape, dtype, out, accumulate, stream):
    if dy.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"dy: bfloat16 or float16 is needed, not {dy.dtype}")
    ldy = _matrix(dy, "dy", dy.dtype)
    ldc = _matrix(codes, "codes", torch.int8)
    M, N = dy.shape
    code_rows, K = codes.shape
    _vector(scales, "scales", torch.float32, (code_rows,))
    with _on(dy, stream):
        if out is None:
            if accumulate:
                raise ValueError("accumulate: needs out")
            out = _new(shape, dy.dtype if dtype is None else dtype, dy.device)
        if out.dtype not in (torch.float32, dy.dtype):
            raise TypeError(f"the gradient is float32 or of dy's type, not {out.dtype}")
        ldo = _matrix(out, "out", out.dtype, shape)
        _same_device(dy, codes, scales, out)
        aligned = dy.data_ptr() % 16 == 0 and ldy % 8 == 0
        need = C.c_size_t()
        _call(lib().fmm_int8_grad_workspace_bytes(code_rows, K, M, N, int(aligned), C.byref(need)), "fmm_int8_grad_workspace_bytes")
        workspace = _new((need.value,), torch.uint8, dy.device)
        tail = (workspace.data_ptr(), need.value, fmm._stream_ptr(None))
        head = (dy.data_ptr(), _TYPES[dy.dtype], ldy, codes.data_ptr(), ldc, scales.data_ptr(), M, N, K, out.data_ptr(), _TYPES[out.dtype], ldo)
        if what == "fmm_int8_grad_weight":
            _call(lib().fmm_int8_grad_weight(*head, int(accumulate), *tail), what)
        else:
            _call(lib().fmm_int8_grad_input(*head, *tail), what)
    return out


def grad_weight(dy, codes, scales, dtype=torch.float32, out=None, accumulate=False, stream=None):
    """Gradient of matmul's b: dy^T (M x N, 16-bit) times the activations that codes (M x K) and scales stand for: N x K in
    `dtype` (float32 or dy's type).  With accumulate it is added to out."""
    if dy.dim() == 2 and codes.dim() == 2 and codes.shape[0] != dy.shape[0]:
        raise ValueError(f"dy and codes have {dy.shape[0]} and {codes.shape[0]} rows")
    return _grad("fmm_int8_grad_weight", dy, codes, scales, (dy.shape[-1], codes.shape[-1]), dtype, out, accumulate, stream)


def grad_input(dy, codes, scales, dtype=None, out=None, stream=None):
    """Gradient of matmul's a: dy (M x N, 16-bit) times the weight that codes (N x K) and scales stand for: M x K in `dtype`
    (float32 or dy's type, the default)."""
    if dy.dim() == 2 and codes.dim() == 2 and codes.shape[0] != dy.shape[1]:
        raise ValueError(f"dy has {dy.shape[1]} columns, codes {codes.shape[0]} rows")
    return _grad("fmm_int8_grad_input", dy, codes, scales, (dy.shape[0], codes.shape[-1]), dtype, out, False, stream)


def status():
    """Status and location code of the current device's product kernels: (0, 0) unless a bounded wait gave up.  Synchronises."""
    code = C.c_int()
    return lib().fmm_int8_status(C.byref(code)), code.value


def status_clear():
    _call(lib().fmm_int8_status_clear(), "fmm_int8_status_clear")
