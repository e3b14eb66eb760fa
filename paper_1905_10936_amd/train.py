"""Python binding of what else a worker's step is made of (include/ef.h): the gated feed-forward block, drawing tokens from
logits, and clipping a gradient's tensors into the worker's flat row.

Argument marshalling only, with the conventions of layers.py; every tensor has to be on the current device.
"""
import ctypes
import sys

import torch

from . import EF_ERR_NULL, _check, _f32, _ptr, _stream_ptr, lib
from .layers import _TYPES, _act, _handle, _key, _matrix, _one_of, _required, _rows, _type, _vector

EF_GATE_SILU, EF_GATE_GELU = 0, 1
# what csrc/ef_binding.cpp marshals, in the order of its TrainEntries
NATIVE_CALLS = ("ef_gated_forward", "ef_gated_backward", "ef_sample_tokens", "ef_grad_clip")
_package = sys.modules[__package__]     # whose _native is the binding, once it is loaded


def declare(L):
    """Argument types of the entry points this module calls."""
    vp, i64, c_int, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    for name, args in (
            ("ef_gated_forward", [i64, i64, i64, c_int, vp, i64, vp, i64, c_int, vp, i64, vp, i64, vp, vp]),
            ("ef_gated_backward", [vp, i64, i64, i64, c_int, vp, i64, vp, i64, vp, i64, c_int, vp, i64, vp, i64, vp]),
            ("ef_sample_tokens", [vp, i64, i64, c_int, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]),
            ("ef_grad_clip", [vp, c_int, i64, vp, vp, vp, f32, vp, i64, vp, vp]), ("ef_gated_kernels", [c_int, c_int, c_int])):
        getattr(L, name).restype = c_int
        getattr(L, name).argtypes = args


def _here(*tensors):
    """The call goes to the current device's stream."""
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() != torch.cuda.current_device():
            raise TypeError("a tensor is on cuda:%d, the current device is cuda:%d" % (t.get_device(), torch.cuda.current_device()))


def ef_gated_forward(x, w, gate, pre, z, act, stream=None):
    """z [rows][inner] <- act(x Wg^T) * (x Wu^T) with w = [Wg; Wu], 2 inner rows; gate: EF_GATE_SILU or EF_GATE_GELU.  pre [rows][2 inner] <-
    both projections, act <- checkpoint of z; any of the outputs but one may be None."""
    rc = _package._native.gated_forward(x, w, gate, pre, z, act, stream)
    if rc is not None:
        return _check(rc)
    rows, width = _rows(x, "x")
    both = _rows(w, "w")[0]
    if both % 2 or _rows(w, "w")[1] != width:
        raise TypeError("w must have 2 inner rows of %d" % width)
    _here(x, w, pre, z, act)
    _required(rows, w, _one_of(pre, z, act))
    (xp, xs), (wp, ws) = _matrix(x, (rows, width), x.dtype, "x"), _matrix(w, (both, width), x.dtype, "w")
    (pp, ps), (zp, zs) = _matrix(pre, (rows, both), x.dtype, "pre"), _matrix(z, (rows, both // 2), x.dtype, "z")
    _check(lib().ef_gated_forward(rows, width, both // 2, _type(x, "x"), xp, xs, wp, ws, int(gate), pp, ps, zp, zs, _act(act, rows, both // 2),
                                  _stream_ptr(stream)))


def ef_gated_backward(workspace, dz, pre, w, gate, dpre, dx, stream=None):
    """dpre [rows][2 inner] <- gradient of both projections from dz [rows][inner] and what the forward pass left in pre (dpre may be pre);
    dx [rows][width] (or None) <- the input's.  The weights' gradient: ef_weight_grad(workspace, dpre, checkpoint of x, ...)."""
    rc = _package._native.gated_backward(_key(workspace), dz, pre, w, gate, dpre, dx, stream)
    if rc is not None:
        return _check(rc)
    rows, inner = _rows(dz, "dz")
    wrows, width = _rows(w, "w")
    if wrows != 2 * inner:
        raise TypeError("w must have %d rows" % (2 * inner))
    _here(dz, pre, w, dpre, dx)
    _required(rows, pre, dpre)
    (zp, zs), (pp, ps) = _matrix(dz, (rows, inner), dz.dtype, "dz"), _matrix(pre, (rows, 2 * inner), dz.dtype, "pre")
    (wp, ws), (gp, gs) = _matrix(w, (wrows, width), dz.dtype, "w"), _matrix(dpre, (rows, 2 * inner), dz.dtype, "dpre")
    xp, xs = _matrix(dx, (rows, width), dz.dtype, "dx")
    _check(lib().ef_gated_backward(_handle(workspace), rows, width, inner, _type(dz, "dz"), zp, zs, pp, ps, wp, ws, int(gate), gp, gs, xp, xs,
                                   _stream_ptr(stream)))


def ef_sample_tokens(workspace, logits, uniform, temperature, top_k, top_p, min_p, tokens, logp, stream=None):
    """tokens int64 [rows] <- drawn from softmax(logits / temperature), filtered by top_k (int32), top_p and min_p (float32), with uniform
    (float32) in [0, 1); logp float32 [rows] (or None) <- their log-probabilities under softmax(logits).  The settings are vectors of a number a row, or
    None."""
    rc = _package._native.sample_tokens(_key(workspace), logits, uniform, temperature, top_k, top_p, min_p, tokens, logp, stream)
    if rc is not None:
        return _check(rc)
    shape = _rows(logits, "logits")
    n = shape[0]
    _here(logits, uniform, temperature, top_k, top_p, min_p, tokens, logp)
    _required(n, uniform, tokens)
    lp, ls = _matrix(logits, shape, logits.dtype, "logits")
    _check(lib().ef_sample_tokens(_handle(workspace), n, shape[1], _type(logits, "logits"), lp, ls, _vector(uniform, n, _f32, "uniform"),
                                  _vector(temperature, n, _f32, "temperature"), _vector(top_k, n, torch.int32, "top_k"),
                                  _vector(top_p, n, _f32, "top_p"), _vector(min_p, n, _f32, "min_p"), _vector(tokens, n, torch.int64, "tokens"),
                                  _vector(logp, n, _f32, "logp"), _stream_ptr(stream)))


def ef_grad_clip(workspace, grads, max_norm, flat, norm, stream=None):
    """norm float32 [workers] <- norms over each worker's tensors; flat (float32, a row a worker, or None: the tensors themselves) <- the tensors one
    after the other, scaled to max_norm where the norm is above it.  grads: a worker's tensors, or a list of such lists; every worker's have the same
    sizes and types."""
    rc = _package._native.grad_clip(_key(workspace), grads, max_norm, flat, norm, stream)
    if rc is not None:
        return _check(rc)
    if not isinstance(grads, (list, tuple)):
        raise TypeError("grads must be a list of tensors, or a list of such lists")
    lists = grads if grads and isinstance(grads[0], (list, tuple)) else [grads]
    sizes, types, pointers = [], [], []
    for w, worker in enumerate(lists):
        if not isinstance(worker, (list, tuple)) or len(worker) != len(lists[0]):
            raise TypeError("every worker must have the same number of tensors")
        for i, t in enumerate(worker):
            if not isinstance(t, torch.Tensor) or t.dtype not in _TYPES:
                raise TypeError("gradients must be float32 or bfloat16 tensors")
            _here(t)
            pointers.append(_ptr(t, t.dtype, "a gradient"))
            if w == 0:
                sizes.append(t.numel())
                types.append(_TYPES[t.dtype])
            elif sizes[i] != t.numel() or types[i] != _TYPES[t.dtype]:
                raise TypeError("every worker's tensors must have the same sizes and types")
    n, total = len(lists), sum(sizes)
    fp, fs = None, 0
    if flat is not None:
        shape = _rows(flat, "flat")
        if shape[0] != n or shape[1] < total:
            raise TypeError("flat must have %d rows of at least %d" % (n, total))
        fp, fs = _matrix(flat, shape, _f32, "flat")
    if norm is None:
        _check(EF_ERR_NULL)
    _here(flat, norm)
    _check(lib().ef_grad_clip(_handle(workspace), n, len(sizes), (ctypes.c_void_p * max(1, len(pointers)))(*pointers),
                              (ctypes.c_int64 * max(1, len(sizes)))(*sizes), (ctypes.c_int * max(1, len(types)))(*types), float(max_norm), fp, fs,
                              _vector(norm, n, _f32, "norm"), _stream_ptr(stream)))
