"""The 8-bit integer layer of libfmm_b200.so: ctypes binding of include/fmm_int8.h (argument checks and marshalling only;
every step runs in the CUDA kernels).

A forward and backward pass of one layer, everything that is kept for the backward pass in 8 bits:

    w, ws = int8.quantize(weight)                                   # (N, K): one scale per output channel
    n = int8.rms_norm(x, gain, residual=r, pow2=True, checkpoint=128)    # hidden rows, their 8-bit norm, a checkpoint
    z = int8.matmul(n.codes, n.scales, w, ws)                       # (M, N)
    ...
    dw = int8.grad_weight(dz, n.codes, n.scales)                    # (N, K)
    dy = int8.grad_input(dz, w, ws)                                 # (M, K)
    dx, dgain = int8.rms_norm_backward(dy, n.checkpoint, n.checkpoint_scales, n.rstd, gain, block=128, dresidual=dh)

Matrices are 2-D CUDA tensors whose columns are contiguous (rows may lie any distance apart); scales and gains are
contiguous.  All tensors of a call are on one device, on whose current stream the work is enqueued, or on `stream`; nothing
is synchronised, and calls may be captured into CUDA graphs.  Outputs are allocated unless they are given; codes get rows
that are a multiple of 16 bytes apart, as `matmul` wants them.  Unsuitable arguments raise TypeError (types, devices) or
ValueError (shapes, strides, blocks), anything that the library refuses raises fmm.FmmError.  Nothing is recorded for autograd,
also of tensors that require a gradient: the gradients are calls of their own.
"""
from __future__ import annotations

import collections
import ctypes as C
import operator
import struct

import torch

from . import fmm

AMAX_DIV_127, POW2 = 0, 1
F32, BF16, F16 = 0, 1, 2
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

EXPORTS = ["fmm_int8_quantize", "fmm_int8_dequantize", "fmm_int8_rms_norm", "fmm_int8_rms_norm_backward_workspace_bytes",
           "fmm_int8_rms_norm_backward", "fmm_int8_matmul", "fmm_int8_grad_weight_workspace_bytes",
           "fmm_int8_grad_input_workspace_bytes", "fmm_int8_grad_weight", "fmm_int8_grad_input", "fmm_int8_product_shape",
           "fmm_int8_force_product_shape", "fmm_int8_status", "fmm_int8_status_clear", "fmm_int8_selftest_bounded_wait"]


class QuantizeArgs(C.Structure):
    """fmm_int8_quantize_t"""
    _fields_ = [("type", C.c_int), ("block", C.c_int), ("scale_mode", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64), ("x", C.c_void_p),
                ("ldx", C.c_int64), ("codes", C.c_void_p), ("ldc", C.c_int64), ("scales", C.c_void_p)]


class DequantizeArgs(C.Structure):
    """fmm_int8_dequantize_t"""
    _fields_ = [("type", C.c_int), ("block", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64), ("codes", C.c_void_p), ("ldc", C.c_int64),
                ("scales", C.c_void_p), ("x", C.c_void_p), ("ldx", C.c_int64)]


class MatmulArgs(C.Structure):
    """fmm_int8_matmul_t"""
    _fields_ = [("type", C.c_int), ("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("a", C.c_void_p), ("lda", C.c_int64), ("a_scales", C.c_void_p),
                ("b", C.c_void_p), ("ldb", C.c_int64), ("b_scales", C.c_void_p), ("bias", C.c_void_p), ("c", C.c_void_p), ("ldc", C.c_int64)]


class GradArgs(C.Structure):
    """fmm_int8_grad_t"""
    _fields_ = [("type", C.c_int), ("out_type", C.c_int), ("accumulate", C.c_int), ("rounded", C.c_int), ("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64),
                ("dy", C.c_void_p), ("ldy", C.c_int64), ("codes", C.c_void_p), ("ldc", C.c_int64), ("scales", C.c_void_p), ("out", C.c_void_p),
                ("ldo", C.c_int64)]


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


class ProductShape(C.Structure):
    """fmm_int8_product_shape_t; iterates as (kernel, columns, k_shares)."""
    _fields_ = [("kernel", C.c_int), ("columns", C.c_int), ("k_shares", C.c_int)]

    def __iter__(self):
        return iter((self.kernel, self.columns, self.k_shares))


KERNEL_PAIRS, KERNEL_CLUSTER, KERNEL_FEW_TOKENS = 1, 2, 3
MATMUL, GRAD_WEIGHT, GRAD_INPUT = 0, 1, 2


def _packer(kind):
    """pack() of the same bytes as kind(*fields): a quarter of the time that filling a ctypes structure takes, and a new object
    for every call, so that threads do not share one.  Addresses are 0, not None."""
    code = {C.c_int: "i", C.c_int64: "q", C.c_double: "d", C.c_void_p: "P"}
    s = struct.Struct("@" + "".join(code[c] for _, c in kind._fields_))
    assert s.size == C.sizeof(kind)
    return s.pack


_quantize_args, _dequantize_args, _matmul_args = _packer(QuantizeArgs), _packer(DequantizeArgs), _packer(MatmulArgs)
_grad_args, _norm_args, _back_args = _packer(GradArgs), _packer(RmsNormArgs), _packer(RmsNormBackwardArgs)

_lib = None


def lib():
    global _lib
    if _lib is None:
        L = fmm.lib()
        ptr, i64, size = C.c_void_p, C.c_int64, C.c_size_t
        for name in ("quantize", "dequantize", "rms_norm", "matmul", "grad_weight_workspace_bytes", "grad_input_workspace_bytes"):
            getattr(L, "fmm_int8_" + name).argtypes = [ptr, ptr]
        for name in ("rms_norm_backward", "grad_weight", "grad_input"):
            getattr(L, "fmm_int8_" + name).argtypes = [ptr, ptr, size, ptr]
        L.fmm_int8_rms_norm_backward_workspace_bytes.argtypes = [i64, i64, ptr]
        L.fmm_int8_status.argtypes = [ptr]
        L.fmm_int8_product_shape.argtypes = [C.c_int, i64, i64, i64, C.c_int, ptr]
        L.fmm_int8_force_product_shape.argtypes = [ptr]
        L.fmm_int8_selftest_bounded_wait.argtypes = [i64, ptr]
        _lib = L
    return _lib


# ------------------------------------------------------------------------------------------------ checks
# (The calls of one token are bound by what Python does for them: a microsecond each for a context manager, an allocation, a few
# checks.  So the checks read every attribute once, devices are compared by number, and the usual device and stream take no context.)
def _device(t):
    """Number of the CUDA device that a call's first tensor is on."""
    try:
        device = t.get_device()
    except AttributeError:
        raise TypeError("a CUDA tensor is needed") from None
    if device < 0:
        raise TypeError("a CUDA tensor is needed")
    return device


def _suits(t, name, dtype, device):
    try:
        where = t.get_device()
    except AttributeError:
        raise TypeError(f"{name}: a CUDA tensor is needed") from None
    if where != device:
        raise TypeError(f"{name}: on {t.device} in a call on cuda:{device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {dtype} is needed, not {t.dtype}")


def _matrix(t, name, dtype, device, shape=None):
    """A 2-D tensor with contiguous columns; its row distance."""
    _suits(t, name, dtype, device)
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise ValueError(f"{name}: shape {tuple(size)}, {'two dimensions are' if shape is None else f'{tuple(shape)} is'} needed")
    rows, cols = size
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: columns are not contiguous")
    if ld < cols or ld < 1:
        if rows > 1 and cols > 0:
            raise ValueError(f"{name}: rows overlap or run backwards")
        ld = max(cols, 1)
    return ld


def _vector(t, name, dtype, device, shape):
    _suits(t, name, dtype, device)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor of shape {shape} is needed, not {tuple(t.shape)}")


def _float_type(dtype, name):
    kind = _TYPES.get(dtype)
    if kind is None:
        raise TypeError(f"{name}: float32, bfloat16 or float16 is needed, not {dtype}")
    return kind


def _block(block, name="block"):
    try:
        block = operator.index(block)
    except TypeError:
        raise TypeError(f"{name}: 0, 32 or 128 is needed, not {block!r}") from None
    if block not in (0, 32, 128):
        raise ValueError(f"{name}: 0, 32 or 128 is needed, not {block}")
    return block


def _number(x, name):
    try:
        return float(x)
    except (TypeError, ValueError):
        raise TypeError(f"{name}: a number is needed, not {x!r}") from None


def _scale_shape(rows, cols, block):
    return (rows, -(-cols // block)) if block else (rows,)


def _elsewhere(device, stream):
    """None where a call can run on the current device and stream, else the context in which it can."""
    if stream is not None:
        if not isinstance(stream, torch.cuda.Stream):
            raise TypeError(f"stream: a torch.cuda.Stream is needed, not {stream!r}")
        if stream.device.index != device:
            raise TypeError(f"a stream of {stream.device} for tensors on cuda:{device}")
        return torch.cuda.stream(stream)
    return None if device == _current_device() else torch.cuda.device(device)


# (torch.cuda.current_stream builds an object; the raw handle is what is needed)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _new_codes(rows, cols, like):
    """Codes whose rows are a multiple of 16 bytes apart, on like's device."""
    if cols % 16 == 0:
        return like.new_empty((rows, cols), dtype=torch.int8)
    return like.new_empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8)[:, :cols]


def _new_like(t):
    """A dense matrix of t's shape and type (0.5 us less where t is dense itself)."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _call(status, what):
    if status:
        fmm._check(status, what)


_needs = {}


def _need(name, key, *args):
    """Workspace bytes by the library's function of that name (remembered by device and by what they depend on)."""
    key = (name, _current_device(), key)
    need = _needs.get(key)
    if need is None:
        b = C.c_size_t()
        _call(getattr(lib(), name)(*args, C.byref(b)), name)
        if len(_needs) >= 1024:
            _needs.clear()
        need = _needs[key] = b.value
    return need


# ------------------------------------------------------------------------------------------------ operators
def quantize(x, block=0, pow2=False, out=None, stream=None):
    """Codes and scales of x (rows x cols): one scale per row, or per block of 32 or 128 columns of a row; with pow2 each is
    a power of two.  out: (codes, scales) to write to."""
    device = _device(x)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return quantize(x, block, pow2, out)
    kind = _float_type(x.dtype, "x")
    ldx = _matrix(x, "x", x.dtype, device)
    rows, cols = x.shape
    block = _block(block)
    shape = _scale_shape(rows, cols, block)
    if out is None:
        codes, scales = _new_codes(rows, cols, x), x.new_empty(shape, dtype=torch.float32)
        ldc = codes.stride(0) or 1
    else:
        codes, scales = out
        ldc = _matrix(codes, "codes", torch.int8, device, (rows, cols))
        _vector(scales, "scales", torch.float32, device, shape)
    a = _quantize_args(kind, block, POW2 if pow2 else AMAX_DIV_127, rows, cols, x.data_ptr(), ldx, codes.data_ptr(), ldc, scales.data_ptr())
    _call((_lib or lib()).fmm_int8_quantize(a, _stream(device)), "fmm_int8_quantize")
    return codes, scales


def dequantize(codes, scales, block=0, dtype=torch.bfloat16, out=None, stream=None):
    """The values that codes stand for, code * scale, in `dtype` (or out's type)."""
    device = _device(codes)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return dequantize(codes, scales, block, dtype, out)
    ldc = _matrix(codes, "codes", torch.int8, device)
    rows, cols = codes.shape
    block = _block(block)
    _vector(scales, "scales", torch.float32, device, _scale_shape(rows, cols, block))
    if out is None:
        kind, out, ldx = _float_type(dtype, "dtype"), codes.new_empty((rows, cols), dtype=dtype), cols
    else:
        kind = _float_type(out.dtype, "out")
        ldx = _matrix(out, "out", out.dtype, device, (rows, cols))
    a = _dequantize_args(kind, block, rows, cols, codes.data_ptr(), ldc, scales.data_ptr(), out.data_ptr(), ldx)
    _call((_lib or lib()).fmm_int8_dequantize(a, _stream(device)), "fmm_int8_dequantize")
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
    device = _device(x)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return rms_norm(x, gain, residual, eps, pow2, checkpoint, hidden)
    dtype = x.dtype
    kind = _float_type(dtype, "x")
    ldx = _matrix(x, "x", dtype, device)
    rows, cols = x.shape
    _vector(gain, "gain", dtype, device, (cols,))
    eps, checkpoint = _number(eps, "eps"), _block(checkpoint, "checkpoint")
    ldr = ldh = ldk = 0
    at_residual = at_hidden = at_kept = at_kept_scales = 0
    if residual is not None:
        ldr = _matrix(residual, "residual", dtype, device, (rows, cols))
        if hidden is None:
            hidden, ldh = _new_like(x), cols
        else:
            ldh = _matrix(hidden, "hidden", dtype, device, (rows, cols))
        at_residual, at_hidden = residual.data_ptr(), hidden.data_ptr()
    elif hidden is not None:
        raise ValueError("hidden: written with a residual only")
    codes = _new_codes(rows, cols, x)
    scales, rstd = x.new_empty((rows,), dtype=torch.float32), x.new_empty((rows,), dtype=torch.float32)
    kept = kept_scales = None
    if checkpoint:
        kept = _new_codes(rows, cols, x)
        kept_scales = x.new_empty(_scale_shape(rows, cols, checkpoint), dtype=torch.float32)
        at_kept, ldk, at_kept_scales = kept.data_ptr(), kept.stride(0), kept_scales.data_ptr()
    a = _norm_args(kind, POW2 if pow2 else AMAX_DIV_127, checkpoint, rows, cols, eps, x.data_ptr(), ldx, at_residual, ldr, gain.data_ptr(),
                    at_hidden, ldh, codes.data_ptr(), codes.stride(0), scales.data_ptr(), rstd.data_ptr(), at_kept, ldk, at_kept_scales)
    _call((_lib or lib()).fmm_int8_rms_norm(a, _stream(device)), "fmm_int8_rms_norm")
    return Norm(x if residual is None else hidden, codes, scales, rstd, kept, kept_scales)


def rms_norm_backward(dy, checkpoint, checkpoint_scales, rstd, gain, block=128, dresidual=None, dx=None, stream=None):
    """(dx, dgain) of the norm, from the checkpoint of its hidden rows and their rstd.  dx, the gradient of x and of residual,
    includes dresidual, the gradient that reaches the hidden rows elsewhere; it may be dy or dresidual.  dgain is float32."""
    device = _device(dy)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return rms_norm_backward(dy, checkpoint, checkpoint_scales, rstd, gain, block, dresidual, dx)
    dtype = dy.dtype
    kind = _float_type(dtype, "dy")
    ldy = _matrix(dy, "dy", dtype, device)
    rows, cols = dy.shape
    ldk = _matrix(checkpoint, "checkpoint", torch.int8, device, (rows, cols))
    block = _block(block)
    _vector(checkpoint_scales, "checkpoint_scales", torch.float32, device, _scale_shape(rows, cols, block))
    _vector(rstd, "rstd", torch.float32, device, (rows,))
    _vector(gain, "gain", dtype, device, (cols,))
    ldr = at_dresidual = 0
    if dresidual is not None:
        ldr, at_dresidual = _matrix(dresidual, "dresidual", dtype, device, (rows, cols)), dresidual.data_ptr()
    if dx is None:
        dx, ldx = _new_like(dy), cols
    else:
        ldx = _matrix(dx, "dx", dtype, device, (rows, cols))
    dgain = dy.new_empty((cols,), dtype=torch.float32)
    need = _need("fmm_int8_rms_norm_backward_workspace_bytes", (rows, cols), rows, cols)
    workspace = dy.new_empty((need,), dtype=torch.uint8)
    a = _back_args(kind, block, rows, cols, dy.data_ptr(), ldy, checkpoint.data_ptr(), ldk, checkpoint_scales.data_ptr(), rstd.data_ptr(),
                            gain.data_ptr(), at_dresidual, ldr, dx.data_ptr(), ldx, dgain.data_ptr())
    _call((_lib or lib()).fmm_int8_rms_norm_backward(a, workspace.data_ptr(), need, _stream(device)), "fmm_int8_rms_norm_backward")
    return dx, dgain


def matmul(a, a_scales, b, b_scales, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """a (M x K codes, a scale per row) times the transpose of b (N x K codes, a scale per row), plus bias (N): M x N in
    `dtype` (or out's type).  The rows of a and b start on 16-byte boundaries; K is at most 131071."""
    device = _device(a)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return matmul(a, a_scales, b, b_scales, bias, dtype, out)
    lda = _matrix(a, "a", torch.int8, device)
    M, K = a.shape
    ldb = _matrix(b, "b", torch.int8, device)
    N = b.shape[0]
    if b.shape[1] != K:
        raise ValueError(f"a and b have {K} and {b.shape[1]} columns")
    # a single row need not be any distance from the next
    if M == 1:
        lda = (K + 15) // 16 * 16
    if N == 1:
        ldb = (K + 15) // 16 * 16
    at_a, at_b = a.data_ptr(), b.data_ptr()
    if (lda | ldb | at_a | at_b) & 15 and M and N and K:
        raise ValueError("a and b: rows have to start on 16-byte boundaries (as those of quantize and rms_norm do)")
    _vector(a_scales, "a_scales", torch.float32, device, (M,))
    _vector(b_scales, "b_scales", torch.float32, device, (N,))
    if out is None:
        kind, out, ldc = _float_type(dtype, "dtype"), a.new_empty((M, N), dtype=dtype), N
    else:
        dtype = out.dtype
        kind = _float_type(dtype, "out")
        ldc = _matrix(out, "out", dtype, device, (M, N))
    if bias is not None:
        _vector(bias, "bias", dtype, device, (N,))
    p = _matmul_args(kind, M, N, K, at_a, lda, a_scales.data_ptr(), at_b, ldb, b_scales.data_ptr(), 0 if bias is None else bias.data_ptr(),
                   out.data_ptr(), ldc)
    _call((_lib or lib()).fmm_int8_matmul(p, _stream(device)), "fmm_int8_matmul")
    return out


def _grad(what, device, dy, codes, scales, shape, dtype, out, accumulate, rounded):
    kind = dy.dtype
    if kind is not torch.bfloat16 and kind is not torch.float16:
        raise TypeError(f"dy: bfloat16 or float16 is needed, not {kind}")
    ldy = _matrix(dy, "dy", kind, device)
    ldc = _matrix(codes, "codes", torch.int8, device)
    M, N = dy.shape
    code_rows, K = codes.shape
    _vector(scales, "scales", torch.float32, device, (code_rows,))
    if out is None:
        if accumulate:
            raise ValueError("accumulate: needs out")
        dtype = kind if dtype is None else dtype
        if dtype is not torch.float32 and dtype is not kind:
            raise TypeError(f"the gradient is float32 or of dy's type, not {dtype}")
        out, ldo = dy.new_empty(shape, dtype=dtype), shape[1]
    else:
        dtype = out.dtype
        if dtype is not torch.float32 and dtype is not kind:
            raise TypeError(f"the gradient is float32 or of dy's type, not {dtype}")
        ldo = _matrix(out, "out", dtype, device, shape)
    at = dy.data_ptr()
    rounded = bool(rounded)
    a = _grad_args(_TYPES[kind], _TYPES[dtype], bool(accumulate), rounded, M, N, K, at, ldy, codes.data_ptr(), ldc, scales.data_ptr(), out.data_ptr(), ldo)
    need = _need(what + "_workspace_bytes", (M, N, K, not (at & 15 or ldy & 7), kind, dtype, rounded), a)
    workspace = dy.new_empty((need,), dtype=torch.uint8)
    call = (_lib or lib()).fmm_int8_grad_weight if what == "fmm_int8_grad_weight" else (_lib or lib()).fmm_int8_grad_input
    _call(call(a, workspace.data_ptr(), need, _stream(device)), what)
    return out


def grad_weight(dy, codes, scales, dtype=torch.float32, out=None, accumulate=False, stream=None, rounded=False):
    """Gradient of matmul's b: dy^T (M x N, 16-bit) times the activations that codes (M x K) and scales stand for: N x K in
    `dtype` (float32 or dy's type).  With accumulate it is added to out.

    The activations count as the numbers of fp32 that they are.  With scales that are powers of two (quantize, rms_norm with
    pow2=True) 16 bits hold them; with others they are multiplied in two or three 16-bit parts, which takes as many times as long.
    With `rounded` in one part, rounded to dy's type: 2^-8 of each at most for bfloat16, 2^-11 for float16."""
    device = _device(dy)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grad_weight(dy, codes, scales, dtype, out, accumulate, rounded=rounded)
    if dy.dim() != 2 or codes.dim() != 2 or codes.shape[0] != dy.shape[0]:
        raise ValueError(f"dy and codes: two dimensions and as many rows are needed, not {tuple(dy.shape)} and {tuple(codes.shape)}")
    return _grad("fmm_int8_grad_weight", device, dy, codes, scales, (dy.shape[1], codes.shape[1]), dtype, out, accumulate, rounded)


def grad_input(dy, codes, scales, dtype=None, out=None, accumulate=False, stream=None, rounded=False):
    """Gradient of matmul's a: dy (M x N, 16-bit) times the weight that codes (N x K) and scales stand for: M x K in `dtype`
    (float32 or dy's type, the default).  With accumulate it is added to out.  Values and `rounded` as for grad_weight; the
    bfloat16 gradient of a bfloat16 dy takes one pass whatever the scales."""
    device = _device(dy)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grad_input(dy, codes, scales, dtype, out, accumulate, rounded=rounded)
    if dy.dim() != 2 or codes.dim() != 2 or codes.shape[0] != dy.shape[1]:
        raise ValueError(f"dy and codes: two dimensions and dy's columns as codes' rows are needed, not {tuple(dy.shape)} and {tuple(codes.shape)}")
    return _grad("fmm_int8_grad_input", device, dy, codes, scales, (dy.shape[0], codes.shape[1]), dtype, out, accumulate, rounded)


def product_shape(which, M, N, K, dtype=torch.float32):
    """The ProductShape that MATMUL, GRAD_WEIGHT or GRAD_INPUT takes on the current device for this size and output type."""
    s = ProductShape()
    _call(lib().fmm_int8_product_shape(which, M, N, K, _float_type(dtype, "dtype"), C.byref(s)), "fmm_int8_product_shape")
    return s


def force_product_shape(kernel=None, columns=256, k_shares=1):
    """Every later call of this host thread takes this shape; without arguments: the library chooses again."""
    s = None if kernel is None else C.byref(ProductShape(kernel, columns, k_shares))
    _call(lib().fmm_int8_force_product_shape(s), "fmm_int8_force_product_shape")


def status():
    """Status and location code of the current device's product kernels: (0, 0) unless a bounded wait gave up.  Synchronises."""
    code = C.c_int()
    return lib().fmm_int8_status(C.byref(code)), code.value


def status_clear():
    _call(lib().fmm_int8_status_clear(), "fmm_int8_status_clear")


def selftest_bounded_wait(limit_ns, stream=None):
    _call(lib().fmm_int8_selftest_bounded_wait(int(limit_ns), fmm._stream_ptr(stream)), "fmm_int8_selftest_bounded_wait")
