"""Python binding of the operators of a worker's forward and backward pass (include/ef.h): RMS norm with an 8-bit
checkpoint, checkpoints on their own, the weight gradient taken from one, and the clipped policy loss.

Argument marshalling only; outputs are tensors the caller owns.  Matrices are 2-D tensors (or 1-D ones: a single row) whose
rows are contiguous, float32 or bfloat16, with any row stride; parameters and their gradients are float32 and may be
slices of a flat vector.
"""
import ctypes
import struct
import sys

import torch

from . import EF_ERR_NULL, _check, _f32, _ptr, _stream_ptr, _u8, lib

EF_TYPE_FP32, EF_TYPE_BF16 = 0, 1
EF_NORM_MAX_WIDTH = 16384
# what csrc/ef_binding.cpp marshals, in the order of its LayerEntries
NATIVE_CALLS = ("ef_act_encode", "ef_act_decode", "ef_norm_forward", "ef_norm_backward", "ef_weight_grad", "ef_token_logp", "ef_policy_loss")
_package = sys.modules[__package__]     # whose _native is the binding, once it is loaded
_TYPES = {torch.float32: EF_TYPE_FP32, torch.bfloat16: EF_TYPE_BF16}


def declare(L):
    """Argument types of the entry points this module calls."""
    vp, i64, c_int, f32, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    for name, result, args in (
            ("ef_act_bytes", size, [i64, i64]), ("ef_act_scales_offset", size, [i64, i64]),
            ("ef_act_encode", c_int, [i64, i64, c_int, vp, i64, vp, vp]),
            ("ef_act_decode", c_int, [i64, i64, vp, c_int, vp, i64, vp]),
            ("ef_norm_forward", c_int, [i64, i64, c_int, vp, i64, vp, i64, vp, f32, vp, i64, vp, i64, vp, vp, vp]),
            ("ef_workspace_create", c_int, [ctypes.POINTER(vp), i64, vp]), ("ef_workspace_destroy", c_int, [vp]),
            ("ef_norm_backward", c_int, [vp, i64, i64, c_int, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, c_int, vp]),
            ("ef_weight_grad", c_int, [vp, i64, i64, i64, c_int, vp, i64, vp, vp, vp, c_int, vp]),
            ("ef_token_logp", c_int, [i64, i64, c_int, vp, i64, vp, vp, vp]),
            ("ef_policy_loss", c_int, [vp, i64, i64, c_int, vp, i64, vp, vp, vp, vp, vp, f32, f32, f32, vp, vp, vp, vp, i64, vp])):
        getattr(L, name).restype = result
        getattr(L, name).argtypes = args


def _rows(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() not in (1, 2):
        raise TypeError("%s must be a 1-D or 2-D torch tensor" % name)
    return (1, t.shape[0]) if t.dim() == 1 else (t.shape[0], t.shape[1])


def _matrix(t, shape, dtype, name):
    """(address, row stride) of a matrix argument; None is none."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA/HIP torch tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if _rows(t, name) != shape:
        raise TypeError("%s must be %d x %d" % ((name,) + shape))
    if shape[1] > 1 and t.stride(-1) != 1:
        raise TypeError("the rows of %s must be contiguous" % name)
    return t.data_ptr(), t.stride(0) if t.dim() == 2 else shape[1]


def _type(t, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in _TYPES:
        raise TypeError("%s must be a float32 or bfloat16 tensor" % name)
    return _TYPES[t.dtype]


def _required(rows, *given):
    """Without rows the library takes null for an empty tensor, so what was not given at all is refused here, as it is with rows."""
    if rows == 0 and any(t is None for t in given):
        _check(EF_ERR_NULL)


def _one_of(*outputs):
    return next((t for t in outputs if t is not None), None)


def _vector(t, n, dtype, name):
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.numel() != n:
        raise TypeError("%s must hold %d entries" % (name, n))
    return _ptr(t, dtype, name)


def ef_act_bytes(rows, width):
    return int(lib().ef_act_bytes(int(rows), int(width)))


def ef_act_scales_offset(rows, width):
    return int(lib().ef_act_scales_offset(int(rows), int(width)))


def _act(t, rows, width, name="act"):
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.numel() != ef_act_bytes(rows, width):
        raise TypeError("%s must hold ef_act_bytes(%d, %d) bytes" % (name, rows, width))
    return _ptr(t, _u8, name)


def ef_act_encode(x, act, stream=None):
    """act: uint8 [ef_act_bytes(rows, width)] <- checkpoint of x [rows][width]."""
    rc = _package._native.act_encode(x, act, stream)
    if rc is not None:
        return _check(rc)
    rows, width = _rows(x, "x")
    _required(rows, act)
    xp, xs = _matrix(x, (rows, width), x.dtype, "x")
    _check(lib().ef_act_encode(rows, width, _type(x, "x"), xp, xs, _act(act, rows, width), _stream_ptr(stream)))


def ef_act_decode(act, y, stream=None):
    """y [rows][width] <- what the checkpoint of such a matrix stands for."""
    rc = _package._native.act_decode(act, y, stream)
    if rc is not None:
        return _check(rc)
    rows, width = _rows(y, "y")
    _required(rows, act)
    yp, ys = _matrix(y, (rows, width), y.dtype, "y")
    _check(lib().ef_act_decode(rows, width, _act(act, rows, width), _type(y, "y"), yp, ys, _stream_ptr(stream)))


def ef_norm_forward(x, residual, weight, eps, h, y, act, rstd, stream=None):
    """h <- x + residual; y <- norm(x + residual) * weight; act <- checkpoint of the norm; rstd float32 [rows].
    residual, weight (float32 [width]) and any of the outputs but one may be None."""
    rc = _package._native.norm_forward(x, residual, weight, eps, h, y, act, rstd, stream)
    if rc is not None:
        return _check(rc)
    shape = _rows(x, "x")
    _required(shape[0], _one_of(h, y, act, rstd))
    (xp, xs), (rp, rs) = _matrix(x, shape, x.dtype, "x"), _matrix(residual, shape, x.dtype, "residual")
    (hp, hs), (yp, ys) = _matrix(h, shape, x.dtype, "h"), _matrix(y, shape, x.dtype, "y")
    _check(lib().ef_norm_forward(shape[0], shape[1], _type(x, "x"), xp, xs, rp, rs, _vector(weight, shape[1], _f32, "weight"), float(eps),
                                 hp, hs, yp, ys, _act(act, *shape), _vector(rstd, shape[0], _f32, "rstd"), _stream_ptr(stream)))


class Workspace:
    """ef_workspace: room for partial results, for calls of up to max_rows rows on the device that was current at
    creation.  Calls that share one must be ordered on the device.  `stream` is not used."""

    def __init__(self, max_rows, stream=None):
        self._h = ctypes.c_void_p()
        self.max_rows = int(max_rows)
        _check(lib().ef_workspace_create(ctypes.byref(self._h), self.max_rows, None))
        self._key = struct.pack("Pq", self._h.value, self.max_rows)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().ef_workspace_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._key = b""

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ef_workspace_create(max_rows, stream=None):
    return Workspace(max_rows, stream)


def ef_workspace_destroy(workspace):
    workspace.close()


def _key(workspace):
    return workspace._key if type(workspace) is Workspace else b""


def _handle(workspace):
    if not isinstance(workspace, Workspace):
        raise TypeError("workspace must be what ef_workspace_create gives")
    return workspace._h


def ef_norm_backward(workspace, dy, act, rstd, weight, dh, dx, dweight, accumulate=False, stream=None):
    """dx <- gradient of the norm's input from dy and (dh, or None) that of its residual path; dweight (float32
    [width], or None) <- or += the weight's."""
    rc = _package._native.norm_backward(_key(workspace), dy, act, rstd, weight, dh, dx, dweight, accumulate, stream)
    if rc is not None:
        return _check(rc)
    shape = _rows(dy, "dy")
    _required(shape[0], act, rstd, dx)
    (gp, gs), (hp, hs) = _matrix(dy, shape, dy.dtype, "dy"), _matrix(dh, shape, dy.dtype, "dh")
    xp, xs = _matrix(dx, shape, dy.dtype, "dx")
    _check(lib().ef_norm_backward(_handle(workspace), shape[0], shape[1], _type(dy, "dy"), gp, gs, _act(act, *shape),
                                  _vector(rstd, shape[0], _f32, "rstd"), _vector(weight, shape[1], _f32, "weight"), hp, hs, xp, xs,
                                  _vector(dweight, shape[1], _f32, "dweight"), int(bool(accumulate)), _stream_ptr(stream)))


def ef_weight_grad(workspace, dz, act, column_scale, dw, accumulate=False, stream=None):
    """dw [out][width] (float32) <- or += dz^T times what act stands for, columns times column_scale (float32 [width], or None)."""
    rc = _package._native.weight_grad(_key(workspace), dz, act, column_scale, dw, accumulate, stream)
    if rc is not None:
        return _check(rc)
    rows, out = _rows(dz, "dz")
    _required(rows, act)
    if not isinstance(dw, torch.Tensor) or dw.dim() != 2 or dw.shape[0] != out:
        raise TypeError("dw must be 2-D, %d x width" % out)
    width = dw.shape[1]
    zp, zs = _matrix(dz, (rows, out), dz.dtype, "dz")
    _check(lib().ef_weight_grad(_handle(workspace), rows, out, width, _type(dz, "dz"), zp, zs, _act(act, rows, width),
                                _vector(column_scale, width, _f32, "column_scale"), _ptr(dw, _f32, "dw"), int(bool(accumulate)),
                                _stream_ptr(stream)))


def ef_token_logp(logits, tokens, logp, stream=None):
    """logp float32 [rows] <- log-probabilities of tokens (int64 [rows]) under softmax(logits [rows][vocab])."""
    rc = _package._native.token_logp(logits, tokens, logp, stream)
    if rc is not None:
        return _check(rc)
    shape = _rows(logits, "logits")
    _required(shape[0], tokens, logp)
    lp, ls = _matrix(logits, shape, logits.dtype, "logits")
    _check(lib().ef_token_logp(shape[0], shape[1], _type(logits, "logits"), lp, ls, _vector(tokens, shape[0], torch.int64, "tokens"),
                               _vector(logp, shape[0], _f32, "logp"), _stream_ptr(stream)))


def ef_policy_loss(workspace, logits, tokens, logp_old, logp_ref, advantage, token_weight, clip_low, clip_high, kl, logp, losses, loss,
                   dlogits, stream=None):
    """Clipped policy loss with a KL term: logp, losses (float32 [rows]), loss (float32 [1]) and dlogits (like logits, or
    logits itself); any of the outputs but one, and logp_old, logp_ref and token_weight, may be None."""
    rc = _package._native.policy_loss(_key(workspace), logits, tokens, logp_old, logp_ref, advantage, token_weight, clip_low, clip_high, kl, logp,
                                       losses, loss, dlogits, stream)
    if rc is not None:
        return _check(rc)
    shape = _rows(logits, "logits")
    n = shape[0]
    _required(n, tokens, advantage, _one_of(logp, losses, loss, dlogits))
    (lp, ls), (gp, gs) = _matrix(logits, shape, logits.dtype, "logits"), _matrix(dlogits, shape, logits.dtype, "dlogits")
    _check(lib().ef_policy_loss(_handle(workspace), n, shape[1], _type(logits, "logits"), lp, ls, _vector(tokens, n, torch.int64, "tokens"),
                                _vector(logp_old, n, _f32, "logp_old"), _vector(logp_ref, n, _f32, "logp_ref"),
                                _vector(advantage, n, _f32, "advantage"), _vector(token_weight, n, _f32, "token_weight"), float(clip_low),
                                float(clip_high), float(kl), _vector(logp, n, _f32, "logp"), _vector(losses, n, _f32, "losses"),
                                _vector(loss, 1, _f32, "loss"), gp, gs, _stream_ptr(stream)))
