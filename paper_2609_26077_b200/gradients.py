"""Norm and clipping of the gradients of all parameters: ctypes binding of include/fmm_gradients.h (argument checks and
marshalling only; every step runs in the CUDA kernels).

    norm = gradients.clip([p.grad for p in parameters], max_norm=1.0)      # in place; a tensor of one number, on the device
    norm = gradients.norm(grads)

Gradients are contiguous CUDA tensors in float32, bfloat16 or float16 (also mixed) on one device, on whose current stream the work is enqueued, or
on `stream`; nothing is synchronised, and calls may be captured into CUDA graphs.  Unsuitable arguments raise TypeError (types, devices) or
ValueError (shapes, strides), anything that the library refuses raises fmm.FmmError.  Nothing is recorded for autograd.
"""
from __future__ import annotations

import ctypes as C
from array import array

import torch

from . import int8
from .fp8 import _usual
from .int8 import _TYPES, _call, _device, _elsewhere, _need, _number, _stream

EXPORTS = ["fmm_gradient_workspace_bytes", "fmm_gradient_norm", "fmm_gradient_clip"]

_lib = None


class ListArgs(C.Structure):
    """fmm_gradients_t"""
    _fields_ = [("count", C.c_int64), ("x", C.c_void_p), ("out", C.c_void_p), ("sizes", C.c_void_p), ("types", C.c_void_p)]


_list_args = int8._packer(ListArgs)


def lib():
    global _lib
    if _lib is None:
        L = int8.lib()
        L.fmm_gradient_workspace_bytes.argtypes = [C.c_int64, C.c_void_p]
        L.fmm_gradient_norm.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.fmm_gradient_clip.argtypes = [C.c_void_p, C.c_double, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
    return _lib


# (The usual call reads the tensors in csrc/calls.cpp, 20 ns each; here it is 45 ns for a property of a tensor.)
_address, _numel, _where, _dense = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous
_dtype = torch.Tensor.dtype.__get__


def _suit(tensors, name, device):
    """The types of the tensors (one, or one for each), all of which are contiguous and on the device; their addresses and sizes."""
    try:
        where = set(map(_where, tensors))
    except TypeError:
        raise TypeError(f"{name}: CUDA tensors are needed") from None
    if where != {device}:
        raise TypeError(f"{name}: on devices {sorted(where)} in a call on cuda:{device}")
    if not all(map(_dense, tensors)):
        raise ValueError(f"{name}: contiguous tensors are needed")
    types = set(map(_dtype, tensors))
    return (types if len(types) == 1 else list(map(_dtype, tensors))), array("q", list(map(_address, tensors))), array("q", list(map(_numel, tensors)))


def _list(tensors, out, device):
    """Bytes of fmm_gradients_t, and what they point to."""
    n = len(tensors)
    dtypes, x, sizes = _suit(tensors, "gradients", device)
    try:
        types = bytes(map(_TYPES.__getitem__, dtypes))
    except KeyError as e:
        raise TypeError(f"gradients: float32, bfloat16 or float16 is needed, not {e.args[0]}") from None
    if len(types) < n:
        types *= n
    to = None
    if out is not None:
        if len(out) != n:
            raise ValueError(f"out: {n} tensors are needed, not {len(out)}")
        out_types, to, out_sizes = _suit(out, "out", device)
        if out_types != dtypes:
            raise TypeError("out: each tensor has to be of its gradient's type")
        if out_sizes != sizes:
            raise ValueError("out: each tensor has to be as large as its gradient")
    kinds = array("B", types)
    return _list_args(n, x.buffer_info()[0], to.buffer_info()[0] if to else 0, sizes.buffer_info()[0], kinds.buffer_info()[0]), (x, to, sizes, kinds)


def _tensors(t, name):
    t = list(t)
    if not t:
        raise ValueError(f"{name}: at least one tensor is needed")
    return t


def norm(gradients, stream=None):
    """The global norm of a list of tensors: sqrt of the sum of the squares of all their numbers, one float32 number on the device."""
    tensors = _tensors(gradients, "gradients")
    if stream is None:
        r = _usual().clip(tensors, None, None)
        if r is not None:
            return r
    device = _device(tensors[0])
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return norm(tensors)
    args, keep = _list(tensors, None, device)
    need = _need("fmm_gradient_workspace_bytes", len(tensors), len(tensors))
    result, workspace = tensors[0].new_empty((), dtype=torch.float32), tensors[0].new_empty((need,), dtype=torch.uint8)
    _call((_lib or lib()).fmm_gradient_norm(args, result.data_ptr(), workspace.data_ptr(), need, _stream(device)), "fmm_gradient_norm")
    return result


def clip(gradients, max_norm, out=None, stream=None):
    """Scales the gradients by min(1, max_norm / norm), in place or into the tensors of `out`, and returns their norm from before (one float32
    number on the device).  Nothing is added to the norm, as torch.nn.utils.clip_grad_norm_ adds 1e-6: a norm of 0 leaves the gradients as they are.  No output may
    share memory with another tensor of the list."""
    tensors, max_norm, out = _tensors(gradients, "gradients"), _number(max_norm, "max_norm"), None if out is None else list(out)
    if stream is None:
        r = _usual().clip(tensors, max_norm, out)
        if r is not None:
            return r
    device = _device(tensors[0])
    where = _elsewhere(device, stream)
    if where is not None:
        with where:
            return clip(tensors, max_norm, out)
    args, keep = _list(tensors, out, device)
    need = _need("fmm_gradient_workspace_bytes", len(tensors), len(tensors))
    result, workspace = tensors[0].new_empty((), dtype=torch.float32), tensors[0].new_empty((need,), dtype=torch.uint8)
    _call((_lib or lib()).fmm_gradient_clip(args, max_norm, result.data_ptr(), workspace.data_ptr(), need, _stream(device)), "fmm_gradient_clip")
    return result
