"""The 8-bit floating-point layer of libfmm_b200.so: binding of include/fmm_fp8.h (argument checks and marshalling only; every step
runs in the CUDA kernels).  The usual calls are made by the module _calls (csrc/calls.cpp), the others from here, through ctypes.  Activations and
weights are e4m3 codes with an fp32 scale for each block of 128.

A forward and backward pass of one layer:

    w, ws = fp8.quantize_weight(weight)                      # (N, K): a scale for each 128 x 128 tile
    q = fp8.quantize_both(x)                                 # (M, K): along the rows for the product, along the columns for dw
    y = fp8.matmul(q.codes, q.scales, w, ws)                 # (M, N); inference takes quantize, which gives the first two only
    ...
    g = fp8.quantize_both(dy)
    dx = fp8.grad_input(g.codes, g.scales, w, ws)            # (M, K)
    dw = fp8.grad_weight(g.column_codes, g.column_scales, q.column_codes, q.column_scales)      # (N, K)

and of a layer of experts, for tokens that are sorted by expert, rows offsets[e] to offsets[e + 1] (int32, on the device) for expert e:

    w, ws = fp8.quantize_weight(weights)                     # (E, N, K)
    q = fp8.quantize_both(x, offsets)
    y = fp8.grouped_matmul(q.codes, q.scales, w, ws, offsets)
    g = fp8.quantize_both(dy, offsets)
    dx = fp8.grouped_grad_input(g.codes, g.scales, w, ws, offsets)
    dw = fp8.grouped_grad_weight(g.column_codes, g.column_scales, q.column_codes, q.column_scales, offsets)     # (E, N, K)

Codes are torch.float8_e4m3fn, a code times its scale being the number.  Scales: along the rows ceil(K / 128) x M, along the columns a row for
each 128 rows x K, of tiles ceil(N / 128) x ceil(K / 128).  The form along the columns has `column_rows` rows, of which a group takes the next
multiple of 128; what is behind the last group in use is not written.  Rows of a grouped call that belong to no group take no part and are not written.

Matrices are 2-D CUDA tensors whose columns are contiguous (rows may lie any distance apart; those of codes start on 16-byte boundaries, as the ones
that are allocated here do, and so may those of scales along rows or columns: where they do not, large products take up to a twentieth longer).  All tensors of
a call are on one device, on whose current stream the work is enqueued, or on `stream`; nothing is synchronised, and calls may be captured into CUDA graphs.  Outputs are allocated unless they are
given; a given one may not overlap an input or another output.  Unsuitable arguments raise TypeError (types, devices) or ValueError (shapes,
strides), anything that the library refuses raises fmm.FmmError.  Nothing is recorded for autograd: the gradients are calls of their own.
"""
from __future__ import annotations

import collections
import ctypes as C
import importlib.util
import operator
import types
import warnings

import torch

from . import build, fmm, int8
from .int8 import _call, _device, _elsewhere, _float_type, _matrix, _packer, _stream, _suits, _vector

BLOCK = 128
MAX_GROUPS = 1024
CODES = torch.float8_e4m3fn

EXPORTS = ["fmm_fp8_column_rows", "fmm_fp8_quantize", "fmm_fp8_quantize_weight", "fmm_fp8_matmul", "fmm_fp8_grad_input", "fmm_fp8_grad_weight",
           "fmm_fp8_force_tile", "fmm_fp8_status", "fmm_fp8_status_clear", "fmm_fp8_selftest_bounded_wait"]


class QuantizeArgs(C.Structure):
    """fmm_fp8_quantize_t"""
    _fields_ = [("type", C.c_int), ("scale_mode", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("groups", C.c_int64), ("offsets", C.c_void_p), ("codes", C.c_void_p), ("ldc", C.c_int64), ("scales", C.c_void_p), ("lds", C.c_int64),
                ("column_codes", C.c_void_p), ("ldcc", C.c_int64), ("column_scales", C.c_void_p), ("ldcs", C.c_int64), ("loose", C.c_int64)]


class QuantizeWeightArgs(C.Structure):
    """fmm_fp8_quantize_weight_t"""
    _fields_ = [("type", C.c_int), ("scale_mode", C.c_int), ("count", C.c_int64), ("rows", C.c_int64), ("cols", C.c_int64), ("x", C.c_void_p),
                ("ldx", C.c_int64), ("step_x", C.c_int64), ("codes", C.c_void_p), ("ldc", C.c_int64), ("step_c", C.c_int64), ("scales", C.c_void_p)]


class ProductArgs(C.Structure):
    """fmm_fp8_product_t"""
    _fields_ = [("type", C.c_int), ("accumulate", C.c_int), ("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("groups", C.c_int64),
                ("offsets", C.c_void_p), ("a", C.c_void_p), ("lda", C.c_int64), ("a_scales", C.c_void_p), ("lda_scales", C.c_int64),
                ("b", C.c_void_p), ("ldb", C.c_int64), ("step_b", C.c_int64), ("b_scales", C.c_void_p), ("ldb_scales", C.c_int64),
                ("bias", C.c_void_p), ("out", C.c_void_p), ("ldo", C.c_int64), ("step_out", C.c_int64), ("loose", C.c_int64), ("tokens", C.c_int64)]


_quantize_args, _weight_args, _product_args = _packer(QuantizeArgs), _packer(QuantizeWeightArgs), _packer(ProductArgs)
_lib = None
_calls = None               # the module of that name, or what stands in for it, once lib() has run


def lib():
    global _lib, _calls
    if _lib is None:
        L = int8.lib()
        for name in ("quantize", "quantize_weight", "matmul", "grad_input", "grad_weight"):
            getattr(L, "fmm_fp8_" + name).argtypes = [C.c_void_p, C.c_void_p]
        L.fmm_fp8_column_rows.argtypes = [C.c_int64, C.c_int64, C.c_void_p]
        L.fmm_fp8_status.argtypes = [C.c_void_p]
        L.fmm_fp8_selftest_bounded_wait.argtypes = [C.c_int64, C.c_void_p]
        _calls, _lib = _load_calls(L), L
    return _lib


def _load_calls(L):
    """The module that makes the usual calls, or, where there is none for this torch and Python, one that leaves them all to the general way."""
    spec = importlib.util.spec_from_file_location(__package__ + "._calls", build.calls_path())
    try:
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError as e:
        warnings.warn(f"calls go through ctypes, which takes the host some microseconds more, as there is no module for torch {torch.__version__} ({e}): "
                      f"`python -m {__package__}.build` makes it", RuntimeWarning, stacklevel=4)
        declines = lambda *a: None
        return types.SimpleNamespace(quantize=declines, product=declines, grad_weight=declines, clip=declines)
    module.bind(*(C.cast(getattr(L, name), C.c_void_p).value for name in (
        "fmm_fp8_quantize", "fmm_fp8_matmul", "fmm_fp8_grad_input", "fmm_fp8_grad_weight", "fmm_gradient_workspace_bytes", "fmm_gradient_norm", "fmm_gradient_clip")))
    return module


def _usual():
    """The module that makes the usual calls; each of its functions returns None for others, which then go the general way."""
    lib()
    return _calls


# ------------------------------------------------------------------------------------------------ checks
def _spaced(t, name, dtype, device, shape, step):
    """A matrix whose rows start on 16-byte boundaries (`step` elements); its row distance."""
    ld = _matrix(t, name, dtype, device, shape)
    rows, cols = t.shape
    if rows <= 1:                                            # a single row need not be any distance from the next
        ld = (cols + step - 1) // step * step or step
    if (ld % step or t.data_ptr() & 15) and rows and cols:
        raise ValueError(f"{name}: rows have to start on 16-byte boundaries (as those that this module allocates do)")
    return ld


def _scales(t, name, device, shape):
    """Scales along rows or columns: the distance of their rows, and whether these start anywhere but on 16-byte boundaries."""
    ld = _matrix(t, name, torch.float32, device, shape)
    if shape[0] <= 1:
        ld = (shape[1] + 3) // 4 * 4 or 4
    return ld, bool(ld % 4 or t.data_ptr() & 15)


def _stack(t, name, dtype, device, groups=None):
    """(ld, step) of a 2-D matrix, or of a 3-D stack of them where `groups` is not None."""
    if groups is None:
        return _matrix(t, name, dtype, device), 0
    _suits(t, name, dtype, device)
    if t.dim() != 3 or t.shape[0] != groups:
        raise ValueError(f"{name}: three dimensions and {groups} groups are needed, not {tuple(t.shape)}")
    _, rows, cols = t.shape
    step, ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name}: columns are not contiguous")
    if rows <= 1:
        ld = max(cols, 1)
    if ld < cols or ld < 1:
        raise ValueError(f"{name}: rows overlap or run backwards")
    if groups > 1 and step < (rows - 1) * ld + cols and rows and cols:
        raise ValueError(f"{name}: matrices overlap or run backwards")
    return ld, (step if groups > 1 else 0)


def _groups(offsets, device):
    _suits(offsets, "offsets", torch.int32, device)
    if offsets.dim() != 1 or offsets.shape[0] < 2 or not offsets.is_contiguous():
        raise ValueError(f"offsets: a contiguous tensor of groups + 1 numbers is needed, not {tuple(offsets.shape)}")
    groups = offsets.shape[0] - 1
    if groups > MAX_GROUPS:
        raise ValueError(f"offsets: {groups} groups, {MAX_GROUPS} at most")
    return groups


def _blocks(n):
    return (n + 127) // 128


def _new_codes(rows, cols, like):
    if cols % 16 == 0:
        return like.new_empty((rows, cols), dtype=CODES)
    return like.new_empty_strided((rows, cols), ((cols + 15) // 16 * 16, 1), dtype=CODES)


def _new_scales(rows, cols, like):
    if cols % 4 == 0:
        return like.new_empty((rows, cols), dtype=torch.float32)
    return like.new_empty_strided((rows, cols), ((cols + 3) // 4 * 4, 1), dtype=torch.float32)


def column_rows(rows, offsets=None):
    """Rows of the form along the columns of `rows` tokens, whatever their distribution over the groups."""
    if offsets is None:
        return _blocks(rows) * 128
    return (rows + 127 * (offsets.shape[0] - 1)) // 128 * 128


# ------------------------------------------------------------------------------------------------ quantization
def _quantize(x, device, pow2, offsets, codes, scales, column_codes, column_scales):
    kind = _float_type(x.dtype, "x")
    ldx = _matrix(x, "x", x.dtype, device)
    rows, cols = x.shape
    groups, at_offsets = (0, 0) if offsets is None else (_groups(offsets, device), offsets.data_ptr())
    p, loose = [0] * 8, False
    if codes is not None:
        lds, loose = _scales(scales, "scales", device, (_blocks(cols), rows))
        p[:4] = codes.data_ptr(), _spaced(codes, "codes", CODES, device, (rows, cols), 16), scales.data_ptr(), lds
    if column_codes is not None:
        padded = column_rows(rows, offsets)
        ldcs, also = _scales(column_scales, "column_scales", device, (padded // 128, cols))
        loose |= also
        p[4:] = column_codes.data_ptr(), _spaced(column_codes, "column_codes", CODES, device, (padded, cols), 16), column_scales.data_ptr(), ldcs
    a = _quantize_args(kind, 1 if pow2 else 0, rows, cols, x.data_ptr(), ldx, groups, at_offsets, *p, loose)
    if rows and cols:
        _call((_lib or lib()).fmm_fp8_quantize(a, _stream(device)), "fmm_fp8_quantize")


def _two_dimensions(x):
    if x.dim() != 2:
        raise ValueError(f"x: shape {tuple(x.shape)}, two dimensions are needed")


def quantize(x, pow2=False, out=None, stream=None):
    """Codes (M x K) and scales (ceil(K / 128) x M) of x along its rows, as matmul and grad_input take them; with pow2 the scales are
    powers of two.  out: (codes, scales) to write to."""
    if out is None and stream is None:
        r = (_calls or _usual()).quantize(x, None, pow2, 1)
        if r is not None:
            return r
    device = _device(x)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return quantize(x, pow2, out)
    _two_dimensions(x)
    rows, cols = x.shape
    codes, scales = (_new_codes(rows, cols, x), _new_scales(_blocks(cols), rows, x)) if out is None else out
    _quantize(x, device, pow2, None, codes, scales, None, None)
    return codes, scales


def quantize_columns(x, offsets=None, pow2=False, out=None, stream=None):
    """Codes (column_rows(M, offsets) x K) and scales (a row for each 128 of those) of x along its columns, as grad_weight takes them."""
    if out is None and stream is None:
        r = (_calls or _usual()).quantize(x, offsets, pow2, 2)
        if r is not None:
            return r
    device = _device(x)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return quantize_columns(x, offsets, pow2, out)
    _two_dimensions(x)
    rows, cols = x.shape
    if out is None:
        if offsets is not None:
            _groups(offsets, device)
        padded = column_rows(rows, offsets)
        out = _new_codes(padded, cols, x), _new_scales(padded // 128, cols, x)
    codes, scales = out
    _quantize(x, device, pow2, offsets, None, None, codes, scales)
    return codes, scales


Forms = collections.namedtuple("Forms", "codes scales column_codes column_scales")


def quantize_both(x, offsets=None, pow2=False, out=None, stream=None):
    """Forms(codes, scales, column_codes, column_scales): both forms of x from one pass over it."""
    if out is None and stream is None:
        r = (_calls or _usual()).quantize(x, offsets, pow2, 3)
        if r is not None:
            return Forms(*r)
    device = _device(x)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return quantize_both(x, offsets, pow2, out)
    _two_dimensions(x)
    rows, cols = x.shape
    if out is None:
        if offsets is not None:
            _groups(offsets, device)
        padded = column_rows(rows, offsets)
        out = Forms(_new_codes(rows, cols, x), _new_scales(_blocks(cols), rows, x), _new_codes(padded, cols, x), _new_scales(padded // 128, cols, x))
    _quantize(x, device, pow2, offsets, *out)
    return Forms(*out)


def quantize_weight(w, pow2=False, out=None, stream=None):
    """Codes and scales of a weight (N x K), or of one for each expert (E x N x K), in tiles of 128 x 128."""
    device = _device(w)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return quantize_weight(w, pow2, out)
    kind = _float_type(w.dtype, "w")
    groups = w.shape[0] if w.dim() == 3 else None
    if groups is not None and groups > MAX_GROUPS:
        raise ValueError(f"w: {groups} experts, {MAX_GROUPS} at most")
    ldx, step_x = _stack(w, "w", w.dtype, device, groups)
    rows, cols = w.shape[-2:]
    shape = (_blocks(rows), _blocks(cols)) if groups is None else (groups, _blocks(rows), _blocks(cols))
    if out is None:
        up = (cols + 15) // 16 * 16
        codes = w.new_empty((*w.shape[:-1], up), dtype=CODES)[..., :cols]
        scales = w.new_empty(shape, dtype=torch.float32)
    else:
        codes, scales = out
        if codes.shape != w.shape:
            raise ValueError(f"codes: shape {tuple(codes.shape)}, {tuple(w.shape)} is needed")
    ldc, step_c = _weight(codes, "codes", device, groups)
    _vector(scales, "scales", torch.float32, device, shape)
    a = _weight_args(kind, 1 if pow2 else 0, 1 if groups is None else groups, rows, cols, w.data_ptr(), ldx, step_x, codes.data_ptr(), ldc, step_c, scales.data_ptr())
    if w.numel():
        _call((_lib or lib()).fmm_fp8_quantize_weight(a, _stream(device)), "fmm_fp8_quantize_weight")
    return codes, scales


def _weight(b, name, device, groups):
    """(ld, step) of a weight's codes, or of one for each group."""
    ld, step = _stack(b, name, CODES, device, groups)
    rows, cols = b.shape[-2:]
    if rows <= 1:
        ld = (cols + 15) // 16 * 16 or 16
    if (ld | step | b.data_ptr()) & 15 and b.numel():
        raise ValueError(f"{name}: rows have to start on 16-byte boundaries (as those of quantize_weight do)")
    return ld, step


# ------------------------------------------------------------------------------------------------ products
def _output(out, dtype, shape, device, like, groups, accumulate):
    if out is None:
        if accumulate:
            raise ValueError("accumulate: needs out")
        return _float_type(dtype, "dtype"), like.new_empty(shape, dtype=dtype), shape[-1], shape[-1] * shape[-2]
    kind = _float_type(out.dtype, "out")
    if out.shape != shape:
        raise ValueError(f"out: shape {tuple(out.shape)}, {tuple(shape)} is needed")
    ldo, step = _stack(out, "out", out.dtype, device, groups)
    return kind, out, ldo, step


def _product(which, a, a_scales, b, b_scales, offsets, bias, dtype, out, accumulate, device):
    groups = None if offsets is None else _groups(offsets, device)
    _suits(a, "a", CODES, device)
    if a.dim() != 2 or b.dim() != (2 if groups is None else 3):
        raise ValueError(f"shapes {tuple(a.shape)} and {tuple(b.shape)}: codes of two dimensions and a weight of {2 if groups is None else 3} are needed")
    M, depth = a.shape
    N, K = b.shape[-2:]
    lda = _spaced(a, "a", CODES, device, None, 16)
    lds, loose = _scales(a_scales, "a_scales", device, (_blocks(depth), M))
    ldb, step_b = _weight(b, "b", device, groups)
    tiles = (_blocks(N), _blocks(K))
    _vector(b_scales, "b_scales", torch.float32, device, tiles if groups is None else (groups, *tiles))
    if which == "fmm_fp8_matmul":
        if depth != K:
            raise ValueError(f"a and b have {depth} and {K} columns")
        shape = (M, N)
    else:
        if depth != N:
            raise ValueError(f"dy has {depth} columns and b {N} rows")
        shape = (M, K)
    kind, out, ldo, _ = _output(out, dtype, shape, device, a, None, accumulate)
    if bias is not None:
        _vector(bias, "bias", out.dtype, device, (N,) if groups is None else (groups, N))
    p = _product_args(kind, bool(accumulate), M, N, K, groups or 0, 0 if offsets is None else offsets.data_ptr(), a.data_ptr(), lda, a_scales.data_ptr(), lds,
                      b.data_ptr(), ldb, step_b, b_scales.data_ptr(), 0, 0 if bias is None else bias.data_ptr(), out.data_ptr(), ldo, 0, loose, 0)
    if M and shape[1]:
        _call(getattr(_lib or lib(), which)(p, _stream(device)), which)
    return out


def matmul(a, a_scales, b, b_scales, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """a (M x K, of quantize) times the transpose of b (N x K, of quantize_weight), plus bias (N): M x N in `dtype` (or out's type)."""
    if stream is None:
        r = (_calls or _usual()).product(1, a, a_scales, b, b_scales, None, bias, dtype, out, False)
        if r is not None:
            return r
    device = _device(a)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return matmul(a, a_scales, b, b_scales, bias, dtype, out)
    return _product("fmm_fp8_matmul", a, a_scales, b, b_scales, None, bias, dtype, out, False, device)


def grad_input(dy, dy_scales, b, b_scales, dtype=torch.bfloat16, out=None, accumulate=False, stream=None):
    """Gradient of matmul's a: dy (M x N, of quantize) times b (N x K, of quantize_weight): M x K in `dtype` (or out's type).  With
    accumulate it is added to out."""
    if stream is None:
        r = (_calls or _usual()).product(2, dy, dy_scales, b, b_scales, None, None, dtype, out, accumulate)
        if r is not None:
            return r
    device = _device(dy)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grad_input(dy, dy_scales, b, b_scales, dtype, out, accumulate)
    return _product("fmm_fp8_grad_input", dy, dy_scales, b, b_scales, None, None, dtype, out, accumulate, device)


def grouped_matmul(a, a_scales, b, b_scales, offsets, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """matmul with a weight for each group of rows: b is E x N x K, bias E x N, and rows offsets[e] to offsets[e + 1] meet b[e]."""
    if stream is None and offsets is not None:
        r = (_calls or _usual()).product(1, a, a_scales, b, b_scales, offsets, bias, dtype, out, False)
        if r is not None:
            return r
    device = _device(a)
    _groups(offsets, device)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grouped_matmul(a, a_scales, b, b_scales, offsets, bias, dtype, out)
    return _product("fmm_fp8_matmul", a, a_scales, b, b_scales, offsets, bias, dtype, out, False, device)


def grouped_grad_input(dy, dy_scales, b, b_scales, offsets, dtype=torch.bfloat16, out=None, accumulate=False, stream=None):
    """grad_input with a weight for each group of rows."""
    if stream is None and offsets is not None:
        r = (_calls or _usual()).product(2, dy, dy_scales, b, b_scales, offsets, None, dtype, out, accumulate)
        if r is not None:
            return r
    device = _device(dy)
    _groups(offsets, device)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grouped_grad_input(dy, dy_scales, b, b_scales, offsets, dtype, out, accumulate)
    return _product("fmm_fp8_grad_input", dy, dy_scales, b, b_scales, offsets, None, dtype, out, accumulate, device)


def _grad_weight(dy, dy_scales, x, x_scales, offsets, dtype, out, accumulate, tokens, device):
    groups = None if offsets is None else _groups(offsets, device)
    _suits(dy, "dy", CODES, device)
    _suits(x, "x", CODES, device)
    if dy.dim() != 2 or x.dim() != 2 or dy.shape[0] != x.shape[0] or dy.shape[0] % 128:
        raise ValueError(f"dy and x: two dimensions and the same number of rows, a multiple of 128, are needed, not {tuple(dy.shape)} and {tuple(x.shape)}")
    M, N = dy.shape
    K = x.shape[1]
    ldy, ldx = _spaced(dy, "dy", CODES, device, None, 16), _spaced(x, "x", CODES, device, None, 16)
    ldys, loose = _scales(dy_scales, "dy_scales", device, (M // 128, N))
    ldxs, also = _scales(x_scales, "x_scales", device, (M // 128, K))
    if tokens is not None:
        tokens = operator.index(tokens)
        if not 0 <= tokens <= M:
            raise ValueError(f"tokens: {tokens}, 0 to {M} is needed")
        if tokens == 0:                                      # no group has any, whatever the offsets say
            M = 0
    shape = (N, K) if groups is None else (groups, N, K)
    kind, out, ldo, step = _output(out, dtype, shape, device, dy, groups, accumulate)
    p = _product_args(kind, bool(accumulate), M, N, K, groups or 0, 0 if offsets is None else offsets.data_ptr(), dy.data_ptr(), ldy, dy_scales.data_ptr(), ldys,
                      x.data_ptr(), ldx, 0, x_scales.data_ptr(), ldxs, 0, out.data_ptr(), ldo, step, loose or also, tokens or 0)
    if N and K:
        _call((_lib or lib()).fmm_fp8_grad_weight(p, _stream(device)), "fmm_fp8_grad_weight")
    return out


def grad_weight(dy, dy_scales, x, x_scales, dtype=torch.float32, out=None, accumulate=False, stream=None):
    """Gradient of matmul's b: the transpose of dy times x, both of quantize_columns: N x K in `dtype` (or out's type).  With accumulate it
    is added to out."""
    if stream is None:
        r = (_calls or _usual()).grad_weight(dy, dy_scales, x, x_scales, None, dtype, out, accumulate)
        if r is not None:
            return r
    device = _device(dy)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grad_weight(dy, dy_scales, x, x_scales, dtype, out, accumulate)
    return _grad_weight(dy, dy_scales, x, x_scales, None, dtype, out, accumulate, None, device)


def grouped_grad_weight(dy, dy_scales, x, x_scales, offsets, dtype=torch.float32, out=None, accumulate=False, stream=None, tokens=None):
    """grad_weight for each group of rows: E x N x K, zeros (or nothing added) where a group has no rows.  tokens: their number, which the forms along the
    columns do not tell, to which offsets beyond it are cut, as the other calls do; without it there must be none."""
    if stream is None and offsets is not None:
        r = (_calls or _usual()).grad_weight(dy, dy_scales, x, x_scales, offsets, dtype, out, accumulate, tokens)
        if r is not None:
            return r
    device = _device(dy)
    _groups(offsets, device)
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return grouped_grad_weight(dy, dy_scales, x, x_scales, offsets, dtype, out, accumulate, tokens=tokens)
    return _grad_weight(dy, dy_scales, x, x_scales, offsets, dtype, out, accumulate, tokens, device)


def force_tile(columns=0, shares=1):
    """Every later product of this host thread takes tiles of 256, 128, 64 or 8 columns (the last two: matmul and grouped_matmul only), whose contraction
    `shares` CTAs share (1 to 4 with 64 and 128); without arguments: the library chooses again."""
    _call(lib().fmm_fp8_force_tile(columns, shares), "fmm_fp8_force_tile")


def status():
    """Status and location code of the current device's kernels of this layer: (0, 0) unless a bounded wait gave up.  Synchronises."""
    code = C.c_int()
    return lib().fmm_fp8_status(C.byref(code)), code.value


def status_clear():
    _call(lib().fmm_fp8_status_clear(), "fmm_fp8_status_clear")


def selftest_bounded_wait(limit_ns, stream=None):
    _call(lib().fmm_fp8_selftest_bounded_wait(int(limit_ns), fmm._stream_ptr(stream)), "fmm_fp8_selftest_bounded_wait")
