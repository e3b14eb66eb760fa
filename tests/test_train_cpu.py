"""What the gated block, the drawing of tokens and clipping refuse, through the C entry points: every check comes before any GPU work, so none is needed, and
no device pointer is followed."""
import ctypes
import inspect
import os
import struct

import pytest
import torch

import paper_1905_10936_amd as ef
from tests.test_layers_cpu import A, B, C, D, E, F, G, INF, NAN, W

OK, NULL, ARG, ALIGN, SIZE = ef.EF_OK, ef.EF_ERR_NULL, ef.EF_ERR_ARG, ef.EF_ERR_ALIGN, ef.EF_ERR_SIZE

CALLS = {
    "ef_gated_forward": dict(rows=10, width=40, inner=30, type=1, x=A, x_stride=40, w=B, w_stride=40, gate=0, pre=C, pre_stride=60, z=D, z_stride=30,
                             act=E, stream=None),
    "ef_gated_backward": dict(ws=W, rows=10, width=40, inner=30, type=1, dz=A, dz_stride=30, pre=B, pre_stride=60, w=C, w_stride=40, gate=1, dpre=D,
                              dpre_stride=60, dx=E, dx_stride=40, stream=None),
    "ef_sample_tokens": dict(ws=W, rows=10, vocab=40, type=1, logits=A, stride=40, uniform=B, temperature=C, top_k=D, top_p=E, min_p=F, tokens=G,
                             logp=G + 4096, stream=None),
}

REFUSALS = [
    ("ef_gated_forward", dict(x=None), NULL), ("ef_gated_forward", dict(w=None), NULL), ("ef_gated_forward", dict(pre=None, z=None, act=None), NULL),
    ("ef_gated_forward", dict(rows=-1), ARG), ("ef_gated_forward", dict(rows=1 << 31), ARG), ("ef_gated_forward", dict(width=0), ARG),
    ("ef_gated_forward", dict(inner=0), ARG), ("ef_gated_forward", dict(type=2), ARG), ("ef_gated_forward", dict(gate=2), ARG),
    ("ef_gated_forward", dict(gate=-1), ARG), ("ef_gated_forward", dict(width=(1 << 24) + 1, x_stride=1 << 25, w_stride=1 << 25), SIZE),
    ("ef_gated_forward", dict(inner=(1 << 24) + 1, pre_stride=1 << 26, z_stride=1 << 25), SIZE), ("ef_gated_forward", dict(x_stride=39), ARG),
    ("ef_gated_forward", dict(w_stride=39), ARG), ("ef_gated_forward", dict(rows=1, w_stride=39), ARG), ("ef_gated_forward", dict(pre_stride=59), ARG),
    ("ef_gated_forward", dict(z_stride=29), ARG), ("ef_gated_forward", dict(z_stride=1 << 62), ARG), ("ef_gated_forward", dict(x=A + 1), ALIGN),
    ("ef_gated_forward", dict(type=0, w=B + 2), ALIGN), ("ef_gated_forward", dict(pre=C + 1), ALIGN), ("ef_gated_forward", dict(z=D + 1), ALIGN),
    ("ef_gated_forward", dict(act=E + 8), ALIGN), ("ef_gated_forward", dict(z=A), ARG), ("ef_gated_forward", dict(z=A + 798), ARG),
    ("ef_gated_forward", dict(pre=B + 4798), ARG), ("ef_gated_forward", dict(act=A + 784), ARG), ("ef_gated_forward", dict(z=C + 2), ARG),
    ("ef_gated_forward", dict(act=C + 1184), ARG),
    ("ef_gated_backward", dict(ws=None), NULL), ("ef_gated_backward", dict(dz=None), NULL), ("ef_gated_backward", dict(pre=None), NULL),
    ("ef_gated_backward", dict(dpre=None), NULL), ("ef_gated_backward", dict(w=None), NULL), ("ef_gated_backward", dict(rows=101), SIZE),
    ("ef_gated_backward", dict(gate=7), ARG), ("ef_gated_backward", dict(type=-1), ARG), ("ef_gated_backward", dict(dz_stride=29), ARG),
    ("ef_gated_backward", dict(pre_stride=59), ARG), ("ef_gated_backward", dict(dpre_stride=59), ARG), ("ef_gated_backward", dict(dx_stride=39), ARG),
    ("ef_gated_backward", dict(w_stride=39), ARG), ("ef_gated_backward", dict(dz=A + 1), ALIGN), ("ef_gated_backward", dict(dx=E + 1), ALIGN),
    ("ef_gated_backward", dict(dpre=B, dpre_stride=61), ARG), ("ef_gated_backward", dict(dpre=B + 2), ARG), ("ef_gated_backward", dict(dpre=A), ARG),
    ("ef_gated_backward", dict(dx=B), ARG), ("ef_gated_backward", dict(dx=C), ARG), ("ef_gated_backward", dict(dx=D + 1198), ARG),
    ("ef_gated_backward", dict(dpre=C + 8), ARG),
    ("ef_sample_tokens", dict(ws=None), NULL), ("ef_sample_tokens", dict(logits=None), NULL), ("ef_sample_tokens", dict(uniform=None), NULL),
    ("ef_sample_tokens", dict(tokens=None), NULL), ("ef_sample_tokens", dict(vocab=0), ARG), ("ef_sample_tokens", dict(vocab=1 << 31, stride=1 << 31), ARG),
    ("ef_sample_tokens", dict(rows=-1), ARG), ("ef_sample_tokens", dict(rows=101), SIZE), ("ef_sample_tokens", dict(type=3), ARG),
    ("ef_sample_tokens", dict(stride=39), ARG), ("ef_sample_tokens", dict(logits=A + 1), ALIGN), ("ef_sample_tokens", dict(tokens=G + 4), ALIGN),
    ("ef_sample_tokens", dict(uniform=B + 2), ALIGN), ("ef_sample_tokens", dict(temperature=C + 1), ALIGN), ("ef_sample_tokens", dict(top_k=D + 2), ALIGN),
    ("ef_sample_tokens", dict(top_p=E + 3), ALIGN), ("ef_sample_tokens", dict(min_p=F + 2), ALIGN), ("ef_sample_tokens", dict(logp=G + 4097), ALIGN),
    ("ef_sample_tokens", dict(tokens=A + 792), ARG), ("ef_sample_tokens", dict(logp=B + 36), ARG), ("ef_sample_tokens", dict(logp=G + 76), ARG),
    ("ef_sample_tokens", dict(tokens=D), ARG), ("ef_sample_tokens", dict(logp=E), ARG),
]


def call(name, **changes):
    args = dict(CALLS[name])
    assert set(changes) <= set(args)
    args.update(changes)
    return getattr(ef.lib(), name)(*args.values())


def clip(grads=(A, B, C, D), sizes=(5, 6), types=(0, 1), workers=2, max_norm=1.0, flat=E, stride=11, norm=F, ws=W, n=None):
    pointers = None if grads is None else (ctypes.c_void_p * max(1, len(grads)))(*grads)
    n = len(sizes or ()) if n is None else n
    return ef.lib().ef_grad_clip(ws, workers, n, pointers, None if sizes is None else (ctypes.c_int64 * max(1, len(sizes)))(*sizes),
                                 None if types is None else (ctypes.c_int * max(1, len(types)))(*types), max_norm, flat, stride, norm, None)


@pytest.mark.parametrize("name,changes,code", REFUSALS, ids=lambda v: str(v) if not isinstance(v, dict) else "-".join(v))
def test_refused(name, changes, code):
    assert call(name, **changes) == code


CLIPS = [(dict(ws=None), NULL), (dict(norm=None), NULL), (dict(grads=None), NULL), (dict(sizes=None, n=2), NULL), (dict(types=None), NULL),
         (dict(grads=(A, None, C, D)), NULL), (dict(workers=0), ARG), (dict(n=-1), ARG), (dict(n=(1 << 20) + 1), ARG), (dict(max_norm=-1.0), ARG),
         (dict(max_norm=NAN), ARG), (dict(max_norm=-INF), ARG), (dict(sizes=(5, -1)), ARG), (dict(types=(0, 2)), ARG), (dict(sizes=(5, (1 << 50) + 1)), SIZE),
         (dict(sizes=(1 << 50, 1 << 50)), SIZE), (dict(stride=10), ARG), (dict(stride=1 << 62), ARG), (dict(flat=E + 2), ALIGN), (dict(norm=F + 1), ALIGN),
         (dict(grads=(A + 2, B, C, D)), ALIGN), (dict(grads=(A, B + 1, C, D)), ALIGN), (dict(flat=A), ARG), (dict(flat=D + 8), ARG), (dict(norm=E + 84), ARG),
         (dict(norm=C), ARG), (dict(flat=None, grads=(A, B, A, D)), ARG), (dict(flat=None, grads=(A, A + 18, C, D)), ARG),
         (dict(flat=None, norm=B + 8), ARG), (dict(grads=(A, B, C, E + 40), workers=2), ARG)]


@pytest.mark.parametrize("changes,code", CLIPS, ids=lambda v: str(v) if not isinstance(v, dict) else "-".join(v))
def test_clip_refused(changes, code):
    assert clip(**changes) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up")
def test_calls_that_are_taken():
    """They get as far as the missing GPU."""
    HIP = ef.EF_ERR_HIP
    assert call("ef_gated_forward") == HIP and call("ef_gated_backward") == HIP and call("ef_sample_tokens") == HIP and clip() == HIP
    assert call("ef_gated_backward", dpre=B) == HIP and call("ef_gated_backward", w=None, dx=None) == HIP
    assert call("ef_gated_forward", rows=1, x_stride=0, pre_stride=0, z_stride=0) == HIP
    # columns side by side in one buffer
    assert call("ef_gated_forward", pre=C, pre_stride=200, z=C + 120, z_stride=200, act=None) == HIP
    assert call("ef_sample_tokens", temperature=None, top_k=None, top_p=None, min_p=None, logp=None) == HIP
    # gradients that are read may be there twice, and side by side; in place they have to be apart
    assert clip(grads=(A, A, A, A)) == HIP and clip(flat=None) == HIP and clip(flat=None, grads=(A, A + 20, C, C + 20)) == HIP
    assert clip(workers=1, grads=(A, B), stride=0) == HIP and clip(sizes=(), types=(), grads=None) == HIP
    assert clip(sizes=(0, 6), grads=(None, B, None, D)) == HIP and clip(max_norm=INF) == HIP and clip(max_norm=0.0) == HIP
    # their fp32 neighbour in memory is not theirs
    assert clip(grads=(E + 88, B, C, D)) == HIP


@pytest.mark.parametrize("name,empty", [("ef_gated_forward", ("x", "pre", "z", "act")), ("ef_gated_backward", ("dz", "pre", "dpre", "dx")),
                                        ("ef_sample_tokens", ("logits", "uniform", "temperature", "top_k", "top_p", "min_p", "tokens", "logp"))])
def test_no_rows(name, empty):
    if torch.cuda.is_available() and "ws" in CALLS[name]:
        pytest.skip("the addresses are made up")
    assert call(name, rows=0, **{k: None for k in empty}) == (ef.EF_ERR_HIP if "ws" in CALLS[name] else OK)
    assert call(name, rows=0, type=9, **{k: None for k in empty}) == ARG


def test_the_binding_says_what_is_wrong():
    x, w, act = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(ef.ef_act_bytes(4, 3), dtype=torch.uint8)
    with pytest.raises(TypeError, match="CUDA"):
        ef.ef_gated_forward(x, w, 0, None, torch.zeros(4, 3), act)
    with pytest.raises(TypeError, match="2 inner rows"):
        ef.ef_gated_forward(x, w[:5], 0, None, torch.zeros(4, 3), act)
    with pytest.raises(TypeError, match="6 rows"):
        ef.ef_gated_backward(None, torch.zeros(4, 3), torch.zeros(4, 6), w[:4], 0, torch.zeros(4, 6), x)
    with pytest.raises(TypeError, match="tensor"):
        ef.ef_sample_tokens(None, [1.0], None, None, None, None, None, None, None)
    for bad in ([1.0], x, [x.half()], [[x], [x, x]], [[x], x]):
        with pytest.raises(TypeError):
            ef.ef_grad_clip(None, bad, 1.0, None, torch.zeros(1))


def test_the_native_calls_leave_what_they_cannot_vouch_for():
    """Without a GPU nothing is taken, whatever its place; the calls have as many arguments as their wrappers."""
    from paper_1905_10936_amd import build, train
    ef.lib()
    if not os.path.exists(build.BINDING):
        pytest.skip("ef_binding.cpp could not be built here")
    t, v, key = torch.zeros(4, 8), torch.zeros(4), struct.pack("Pq", 0, 4)
    k, tokens = torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)
    calls = {"gated_forward": (t, t, 0, t, t, None), "gated_backward": (key, t, t, t, 0, t, t), "sample_tokens": (key, t, v, v, k, v, v, tokens, v),
             "grad_clip": (key, [t, v], 1.0, t, v)}
    assert ["ef_" + name for name in calls] == list(train.NATIVE_CALLS)
    for name, args in calls.items():
        native = getattr(ef._native, name)
        assert len(args) + 1 == len(inspect.signature(getattr(ef, "ef_" + name)).parameters), name
        assert native(*args, None) is None and native(*args) is None and native() is None, name
        assert native(*(None for _ in args), None) is None, name
    for grads in ([], (), [[]], [[], []], [None], [[t], t], [[t], None], 3, "ab"):
        assert ef._native.grad_clip(key, grads, 1.0, t, v, None) is None
    with pytest.raises(TypeError):
        ef._native.bind_train(1)
