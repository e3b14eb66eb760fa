"""What the operators of a worker's forward and backward pass refuse, through the C entry points: every check comes before any GPU work,
so none is needed, and no pointer is followed."""
import ctypes

import pytest
import torch

import paper_1905_10936_amd as ef

OK, NULL, ARG, ALIGN, SIZE = ef.EF_OK, ef.EF_ERR_NULL, ef.EF_ERR_ARG, ef.EF_ERR_ALIGN, ef.EF_ERR_SIZE
A, B, C, D, E, F, G = (k << 40 for k in range(1, 8))        # addresses far apart
NAN, INF = float("nan"), float("inf")


class FakeWorkspace(ctypes.Structure):
    """What the argument checks read of a workspace."""
    _fields_ = [("device", ctypes.c_int), ("max_rows", ctypes.c_int64), ("row_sums", ctypes.c_void_p), ("parts", ctypes.c_void_p),
                ("base", ctypes.c_void_p)]


WS = FakeWorkspace(0, 100, None, None, None)
W = ctypes.addressof(WS)

CALLS = {
    "ef_act_encode": dict(rows=10, width=40, type=1, x=A, x_stride=40, act=B, stream=None),
    "ef_act_decode": dict(rows=10, width=40, act=B, type=1, y=A, y_stride=40, stream=None),
    "ef_norm_forward": dict(rows=10, width=40, type=1, x=A, x_stride=40, residual=B, residual_stride=40, weight=C, eps=1e-6, h=D, h_stride=40, y=E,
                            y_stride=40, act=F, rstd=G, stream=None),
    "ef_norm_backward": dict(ws=W, rows=10, width=40, type=1, dy=A, dy_stride=40, act=B, rstd=C, weight=D, dh=E, dh_stride=40, dx=F, dx_stride=40,
                             dweight=G, accumulate=0, stream=None),
    "ef_weight_grad": dict(ws=W, rows=10, out_width=30, width=40, type=1, dz=A, dz_stride=30, act=B, column_scale=C, dw=D, accumulate=0,
                           stream=None),
    "ef_token_logp": dict(rows=10, vocab=40, type=1, logits=A, stride=40, tokens=B, logp=C, stream=None),
    "ef_policy_loss": dict(ws=W, rows=10, vocab=40, type=1, logits=A, stride=40, tokens=B, logp_old=None, logp_ref=None, advantage=C, token_weight=D,
                           clip_low=0.2, clip_high=0.2, kl=0.1, logp=E, losses=F, loss=G, dlogits=G + 4096, dlogits_stride=40, stream=None),
}

REFUSALS = [
    ("ef_act_encode", dict(x=None), NULL), ("ef_act_encode", dict(act=None), NULL), ("ef_act_encode", dict(rows=-1), ARG),
    ("ef_act_encode", dict(width=0), ARG), ("ef_act_encode", dict(type=2), ARG), ("ef_act_encode", dict(x_stride=39), ARG),
    ("ef_act_encode", dict(x=A + 1), ALIGN), ("ef_act_encode", dict(type=0, x=A + 2), ALIGN), ("ef_act_encode", dict(act=B + 8), ALIGN),
    ("ef_act_encode", dict(act=A), ARG), ("ef_act_encode", dict(act=A + 784), ARG), ("ef_act_encode", dict(rows=1 << 31), ARG),
    ("ef_act_encode", dict(x_stride=1 << 62), ARG), ("ef_act_encode", dict(rows=(1 << 31) - 1, width=1 << 24, x_stride=1 << 24), SIZE),
    ("ef_act_decode", dict(y=None), NULL), ("ef_act_decode", dict(act=None), NULL), ("ef_act_decode", dict(type=-1), ARG),
    ("ef_act_decode", dict(y_stride=3), ARG), ("ef_act_decode", dict(y=B + 640), ARG), ("ef_act_decode", dict(y=A + 1), ALIGN),
    ("ef_norm_forward", dict(x=None), NULL), ("ef_norm_forward", dict(h=None, y=None, act=None, rstd=None), NULL),
    ("ef_norm_forward", dict(width=ef.EF_NORM_MAX_WIDTH + 1), SIZE), ("ef_norm_forward", dict(eps=-1e-6), ARG),
    ("ef_norm_forward", dict(eps=NAN), ARG), ("ef_norm_forward", dict(eps=INF), ARG), ("ef_norm_forward", dict(residual_stride=1), ARG),
    ("ef_norm_forward", dict(h_stride=0), ARG), ("ef_norm_forward", dict(y_stride=-40), ARG), ("ef_norm_forward", dict(weight=C + 2), ALIGN),
    ("ef_norm_forward", dict(rstd=G + 1), ALIGN), ("ef_norm_forward", dict(act=F + 4), ALIGN), ("ef_norm_forward", dict(y=E + 1), ALIGN),
    ("ef_norm_forward", dict(h=E), ARG), ("ef_norm_forward", dict(h=A + 2), ARG), ("ef_norm_forward", dict(h=A, h_stride=41), ARG),
    ("ef_norm_forward", dict(rstd=C + 80), ARG), ("ef_norm_forward", dict(act=A + 16), ARG), ("ef_norm_forward", dict(y=F + 640), ARG),
    ("ef_norm_backward", dict(ws=None), NULL), ("ef_norm_backward", dict(dy=None), NULL), ("ef_norm_backward", dict(act=None), NULL),
    ("ef_norm_backward", dict(rstd=None), NULL), ("ef_norm_backward", dict(dx=None), NULL), ("ef_norm_backward", dict(rows=101), SIZE),
    ("ef_norm_backward", dict(width=ef.EF_NORM_MAX_WIDTH + 1), SIZE), ("ef_norm_backward", dict(dweight=D), ARG),
    ("ef_norm_backward", dict(dx=B + 64), ARG), ("ef_norm_backward", dict(dx=A, dx_stride=50), ARG), ("ef_norm_backward", dict(dweight=G + 2), ALIGN),
    ("ef_norm_backward", dict(dx=E + 2), ARG), ("ef_norm_backward", dict(dy_stride=20), ARG),
    ("ef_weight_grad", dict(ws=None), NULL), ("ef_weight_grad", dict(dz=None), NULL), ("ef_weight_grad", dict(dw=None), NULL),
    ("ef_weight_grad", dict(act=None), NULL), ("ef_weight_grad", dict(rows=101), SIZE), ("ef_weight_grad", dict(width=0), ARG),
    ("ef_weight_grad", dict(out_width=0), ARG), ("ef_weight_grad", dict(out_width=(1 << 24) + 1, dz_stride=1 << 25), SIZE),
    ("ef_weight_grad", dict(width=(1 << 24) + 1), SIZE), ("ef_weight_grad", dict(dz_stride=29), ARG), ("ef_weight_grad", dict(dw=A + 8), ARG),
    ("ef_weight_grad", dict(dw=C - 4), ARG), ("ef_weight_grad", dict(dw=D + 2), ALIGN), ("ef_weight_grad", dict(dz=A + 1), ALIGN),
    ("ef_weight_grad", dict(type=7), ARG),
    ("ef_token_logp", dict(logits=None), NULL), ("ef_token_logp", dict(tokens=None), NULL), ("ef_token_logp", dict(logp=None), NULL),
    ("ef_token_logp", dict(vocab=0), ARG), ("ef_token_logp", dict(vocab=1 << 31, stride=1 << 31), ARG), ("ef_token_logp", dict(tokens=B + 4), ALIGN),
    ("ef_token_logp", dict(logp=A + 40), ARG), ("ef_token_logp", dict(logp=B + 72), ARG), ("ef_token_logp", dict(stride=39), ARG),
    ("ef_policy_loss", dict(ws=None), NULL), ("ef_policy_loss", dict(advantage=None), NULL),
    ("ef_policy_loss", dict(logp=None, losses=None, loss=None, dlogits=None), NULL), ("ef_policy_loss", dict(rows=101), SIZE),
    ("ef_policy_loss", dict(clip_low=-0.1), ARG), ("ef_policy_loss", dict(clip_low=1.5), ARG), ("ef_policy_loss", dict(clip_low=NAN), ARG),
    ("ef_policy_loss", dict(clip_high=-0.1), ARG), ("ef_policy_loss", dict(clip_high=INF), ARG), ("ef_policy_loss", dict(kl=-1.0), ARG),
    ("ef_policy_loss", dict(kl=NAN), ARG), ("ef_policy_loss", dict(dlogits=A, dlogits_stride=48), ARG), ("ef_policy_loss", dict(dlogits=A + 2), ARG),
    ("ef_policy_loss", dict(logp=F), ARG), ("ef_policy_loss", dict(losses=C), ARG), ("ef_policy_loss", dict(dlogits_stride=20), ARG),
    ("ef_policy_loss", dict(loss=G + 2), ALIGN), ("ef_policy_loss", dict(logp_old=D + 1), ALIGN), ("ef_policy_loss", dict(loss=E + 36), ARG),
]


def call(name, **changes):
    args = dict(CALLS[name])
    assert set(changes) <= set(args)
    args.update(changes)
    return getattr(ef.lib(), name)(*args.values())


@pytest.mark.parametrize("name,changes,code", REFUSALS, ids=lambda v: str(v) if not isinstance(v, dict) else "-".join(v))
def test_refused(name, changes, code):
    assert call(name, **changes) == code


@pytest.mark.parametrize("name", ["ef_act_encode", "ef_act_decode", "ef_norm_forward", "ef_token_logp"])
def test_no_rows_is_a_call_that_does_nothing(name):
    assert call(name, rows=0) == OK


def test_rows_side_by_side_in_one_buffer_are_apart():
    """Refused only for what they share: here the columns differ, so the call gets as far as the missing GPU (or, with no rows, nowhere)."""
    side = dict(x=A, x_stride=200, residual=A + 80, residual_stride=200, h=A + 160, h_stride=200, y=A + 240, y_stride=200)
    assert call("ef_norm_forward", **dict(side, y=A + 222)) == ARG
    assert call("ef_norm_forward", **dict(side, y=A + 322)) == ARG      # its last columns are the next row's first
    if not torch.cuda.is_available():
        assert call("ef_norm_forward", **side) == ef.EF_ERR_HIP
        # the same pointer and stride, where a call works in place
        assert call("ef_norm_forward", h=A, y=B) == ef.EF_ERR_HIP


def test_workspace():
    L = ef.lib()
    assert L.ef_workspace_create(None, 1, None) == NULL and L.ef_workspace_destroy(None) == NULL
    p = ctypes.c_void_p()
    assert L.ef_workspace_create(ctypes.byref(p), -1, None) == ARG and L.ef_workspace_create(ctypes.byref(p), 1 << 31, None) == ARG
    assert not p.value
    if not torch.cuda.is_available():
        with pytest.raises(ef.EfError) as e:
            ef.ef_workspace_create(10)
        assert e.value.code == ef.EF_ERR_HIP


def test_sizes_of_checkpoints():
    for rows, width in ((0, 5), (1, 1), (7, 32), (7, 33), (1000, 4096)):
        groups = (width + 31) // 32
        assert ef.ef_act_scales_offset(rows, width) == rows * groups * 32
        assert ef.ef_act_bytes(rows, width) == (rows * groups * 33 + 15) // 16 * 16
    for rows, width in ((-1, 4), (4, 0), (1 << 40, 1 << 40), ((1 << 63) - 1, (1 << 63) - 1)):
        assert ef.ef_act_bytes(rows, width) == 0 and ef.ef_act_scales_offset(rows, width) == 0


def test_the_binding_says_what_is_wrong():
    x, act = torch.zeros(4, 8), torch.zeros(ef.ef_act_bytes(4, 8), dtype=torch.uint8)
    with pytest.raises(TypeError, match="CUDA"):
        ef.ef_act_encode(x, act)
    with pytest.raises(TypeError, match="2-D"):
        ef.ef_act_encode(x[None], act)
    with pytest.raises(TypeError, match="dw must be 2-D"):
        ef.ef_weight_grad(None, x, act, None, torch.zeros(12))
    with pytest.raises(TypeError, match="tensor"):
        ef.ef_token_logp([1.0], None, None)
    x2 = torch.zeros(4, 8)
    with pytest.raises(TypeError, match="CUDA"):
        ef.ef_weight_grad(None, x2, act, None, torch.zeros(8, 8))


def test_the_native_calls_leave_what_they_cannot_vouch_for():
    """Without a GPU nothing is taken, whatever its place; the calls have as many arguments as their wrappers."""
    import inspect
    import os
    import struct

    from paper_1905_10936_amd import build, layers
    ef.lib()
    if not os.path.exists(build.BINDING):
        pytest.skip("ef_binding.cpp could not be built here")
    t, v, act, key = torch.zeros(4, 8), torch.zeros(4), torch.zeros(ef.ef_act_bytes(4, 8), dtype=torch.uint8), struct.pack("Pq", 0, 4)
    tokens = torch.zeros(4, dtype=torch.int64)
    calls = {"act_encode": (t, act), "act_decode": (act, t), "norm_forward": (t, None, None, 0.1, None, t, act, v),
             "norm_backward": (key, t, act, v, None, None, t, None, False), "weight_grad": (key, t, act, None, t, False),
             "token_logp": (t, tokens, v), "policy_loss": (key, t, tokens, v, v, v, v, 0.1, 0.1, 0.1, v, v, None, t)}
    assert ["ef_" + name for name in calls] == list(layers.NATIVE_CALLS)
    for name, args in calls.items():
        call = getattr(ef._native, name)
        assert len(args) + 1 == len(inspect.signature(getattr(ef, "ef_" + name)).parameters), name
        assert call(*args, None) is None and call(*args) is None and call() is None, name
        assert call(*(None for _ in args), None) is None, name
    with pytest.raises(TypeError):
        ef._native.bind_layers(1)
