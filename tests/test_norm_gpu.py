"""RMS norm with the residual's addition and an 8-bit output, and its backward pass, against 64 bits; the gradient also against
differences of the forward pass's formula."""
import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import layer_oracle as oracle
from tests.test_act_gpu import TYPES, checkpoint, parts

pytestmark = pytest.mark.gpu

EPS = 1e-6
UNIT = oracle.EPS
# every team: 16 lanes, a wavefront with 1, 2, 4 pieces, 256 threads with 2 and 4, 512
WIDTHS = [1, 5, 31, 128, 129, 515, 1024, 1031, 2051, 4099, 8200, 16384] + [512, 1540, 2044, 4096, 6145, 12289, 12287]


def half_unit(dtype):
    return 2.0 ** -8 if dtype is torch.bfloat16 else UNIT


def rows_of(rows, n, dtype, seed, sigma=1.0):
    gen = torch.Generator().manual_seed(seed)
    v = torch.randn(rows, n, generator=gen) * sigma
    v[:, ::max(1, n // 5)] *= 12.0
    return v.to(dtype).cuda()


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def check_forward(x, residual, weight, h, y, act, rstd, eps=EPS):
    rows, n = x.shape
    v, want_rstd, xhat, want_y = oracle.norm_forward(f64(x), f64(residual), f64(weight), eps)
    # the sum of squares: at most 32 + 12 additions one after the other; square root, quotients and products round once each
    off = (48 / 2 + 6) * UNIT
    assert np.all(np.abs(f64(rstd) - want_rstd) <= off * want_rstd)
    if h is not None:
        assert np.all(np.abs(f64(h) - v) <= (half_unit(x.dtype) * (1 + 2.0 ** -7) + UNIT) * np.abs(v) + 1e-38)
    if y is not None:
        assert np.all(np.abs(f64(y) - want_y) <= (half_unit(x.dtype) * (1 + 2.0 ** -7) + off + 4 * UNIT) * np.abs(want_y) + 1e-38)
    if act is None:
        return
    codes, scales = parts(act, rows, n)
    # a group's largest magnitude may lie on either side of a threshold, by what xhat is off
    top = np.abs(oracle.groups_of(xhat)).max(-1)
    off += 3 * UNIT
    assert np.all((scales == oracle.scale_bytes(top * (1 - off))) | (scales == oracle.scale_bytes(top * (1 + off))))
    got = oracle.decode(codes, scales, n)
    scale = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, axis=1)[:, :n]
    # half a step of E4M3: 2^-4 of the value, 2^-10 of the scale near zero
    assert np.all(np.abs(got - xhat) <= np.maximum(2.0 ** -4 * np.abs(xhat), 2.0 ** -10 * scale) + 2 * off * np.abs(xhat))
    g = codes.reshape(rows, -1)
    assert not g[:, n:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", WIDTHS)
def test_forward(n, dtype):
    t = TYPES[dtype]
    rows = 37 if n < 4000 else 5
    x, r = rows_of(rows, n, t, n), rows_of(rows, n, t, n + 1)
    w = 1 + 0.2 * torch.randn(n, device="cuda")
    h, y, rstd, act = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), checkpoint(rows, n)
    ef.ef_norm_forward(x, r, w, EPS, h, y, act, rstd)
    check_forward(x, r, w, h, y, act, rstd)
    # without residual and weight, outputs one at a time: the same numbers as together
    y1, act1, rstd1 = torch.empty_like(x), checkpoint(rows, n), torch.empty(rows, device="cuda")
    ef.ef_norm_forward(x, None, None, EPS, None, y1, None, None)
    ef.ef_norm_forward(x, None, None, EPS, None, None, act1, None)
    ef.ef_norm_forward(x, None, None, EPS, None, None, None, rstd1)
    check_forward(x, None, None, None, y1, act1, rstd1)


@pytest.mark.parametrize("dtype", TYPES)
def test_single_rows_in_place_and_strides(dtype):
    t = TYPES[dtype]
    for rows, n in ((1, 1024), (1, 77), (9, 333)):
        x, r = rows_of(rows, n, t, 1), rows_of(rows, n, t, 2)
        w = 1 + 0.2 * torch.randn(n + 3, device="cuda")[3:]         # 4-byte aligned
        h, y, rstd, act = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), checkpoint(rows, n)
        ef.ef_norm_forward(x, r, w, EPS, h, y, act, rstd)
        check_forward(x, r, w, h, y, act, rstd)
        # h over the residual, y over x
        x1, r1, act1 = x.clone(), r.clone(), checkpoint(rows, n)
        ef.ef_norm_forward(x1, r1, w, EPS, r1, x1, act1, None)
        assert torch.equal(r1, h) and torch.equal(x1, y) and torch.equal(act1, act)
        # rows side by side in one buffer, at odd places
        room = torch.full((rows, 4 * n + 9), 3.0, dtype=t, device="cuda")
        xs, rs, hs, ys = (room[:, 1 + k * (n + 1):1 + k * (n + 1) + n] for k in range(4))
        xs.copy_(x)
        rs.copy_(r)
        ef.ef_norm_forward(xs, rs, w, EPS, hs, ys, act1, None)
        assert torch.equal(hs, h) and torch.equal(ys, y) and torch.equal(act1, act)
        assert bool((room[:, 0] == 3).all()) and bool((room[:, -4:] == 3).all()) and bool((room[:, n + 1] == 3).all())
    # one row as a vector
    x = rows_of(1, 515, t, 4)[0]
    y = torch.empty_like(x)
    rstd = torch.empty(1, device="cuda")
    ef.ef_norm_forward(x, None, None, EPS, None, y, None, rstd)
    check_forward(x[None], None, None, None, y[None], None, rstd)


def test_rows_of_zeros_large_numbers_and_nan():
    n = 200
    x = rows_of(6, n, torch.float32, 9)
    x[0] = 0
    x[1] *= 1e15
    x[2] *= 1e-15
    x[3, 7] = float("nan")
    x[4, 190] = float("inf")
    y, act, rstd = torch.empty_like(x), checkpoint(6, n), torch.empty(6, device="cuda")
    ef.ef_norm_forward(x, None, None, EPS, None, y, act, rstd)
    assert bool((y[0] == 0).all()) and abs(float(rstd[0]) - 1e3) < 1e-3
    fine = [0, 1, 2, 5]
    check_forward(x[fine], None, None, None, y[fine], None, rstd[fine])
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[4, 190]))
    assert torch.isfinite(y[fine]).all()
    codes, scales = parts(act, 6, n)
    assert (scales[3] == 255).all() and scales[4, 190 // 32] == 255 and (scales[fine] != 255).all()
    # eps = 0 and a row of zeros: 0 * inf
    ef.ef_norm_forward(x[:1], None, None, 0.0, None, y[:1], None, rstd[:1])
    assert bool(torch.isinf(rstd[0])) and bool(torch.isnan(y[0]).all())


def backward_inputs(rows, n, t, seed, with_dh=True):
    x = rows_of(rows, n, torch.float32, seed)
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    act = checkpoint(rows, n)
    ef.ef_act_encode(x * rstd[:, None], act)
    gen = torch.Generator().manual_seed(seed + 1)
    dy = (torch.randn(rows, n, generator=gen) * 0.1).to(t).cuda()
    dh = (torch.randn(rows, n, generator=gen) * 0.1).to(t).cuda() if with_dh else None
    w = (1 + 0.2 * torch.randn(n, generator=gen)).cuda()
    return dy, act, rstd, w, dh


def check_backward(dy, act, rstd, w, dh, dx, dw, before=None):
    rows, n = dy.shape
    xhat = oracle.decode(*parts(act, rows, n), n)
    want, off, want_dw, off_dw = oracle.norm_backward(f64(dy), xhat, f64(rstd), f64(w), f64(dh))
    assert np.all(np.abs(f64(dx) - want) <= off + half_unit(dy.dtype) * (1 + 2.0 ** -7) * np.abs(want) + 1e-38)
    if dw is not None:
        if before is not None:
            want_dw, off_dw = want_dw + f64(before), off_dw + 2 * UNIT * np.abs(f64(before))
        assert np.all(np.abs(f64(dw) - want_dw) <= off_dw + 1e-38)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", WIDTHS)
def test_backward(n, dtype):
    rows = 301 if n < 4000 else 7
    ws = ef.ef_workspace_create(rows)
    dy, act, rstd, w, dh = backward_inputs(rows, n, TYPES[dtype], n)
    dx, flat = torch.empty_like(dy), torch.full((n + 5,), 2.0, device="cuda")
    dw = flat[3:3 + n]
    ef.ef_norm_backward(ws, dy, act, rstd, w, dh, dx, dw)
    check_backward(dy, act, rstd, w, dh, dx, dw)
    assert bool((flat[:3] == 2).all()) and bool((flat[3 + n:] == 2).all())
    before = dw.clone()
    dx2 = torch.empty_like(dy)
    ef.ef_norm_backward(ws, dy, act, rstd, None, None, dx2, dw, accumulate=True)
    check_backward(dy, act, rstd, None, None, dx2, dw, before)
    # rows alone; in place over dh, over dy
    a, b = dh.clone(), dy.clone()
    ef.ef_norm_backward(ws, dy, act, rstd, w, a, a, None)
    ef.ef_norm_backward(ws, b, act, rstd, w, dh, b, None)
    assert torch.equal(a, dx) and torch.equal(b, dx)


@pytest.mark.parametrize("rows", [1, 3, 2047, 2050, 5000])
def test_backward_over_rows(rows):
    """One team, some without rows, several rows to a team; the same bits every time."""
    n = 96 if rows > 3 else 1100
    ws = ef.ef_workspace_create(rows)
    args = backward_inputs(rows, n, torch.bfloat16, rows)
    dx, dw = torch.empty_like(args[0]), torch.empty(n, device="cuda")
    ef.ef_norm_backward(ws, *args, dx, dw)
    check_backward(*args, dx, dw)
    for _ in range(3):
        dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
        ef.ef_norm_backward(ws, *args, dx2, dw2)
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw)


def test_no_rows_and_a_nan():
    ws = ef.ef_workspace_create(8)
    L = ef.lib()
    some, dw = torch.zeros(64, device="cuda"), torch.full((40,), 3.0, device="cuda")
    p = some.data_ptr()
    assert L.ef_norm_backward(ws._h, 0, 40, 0, p, 40, p, p, None, None, 0, p, 40, dw.data_ptr(), 1, None) == 0
    torch.cuda.synchronize()
    assert bool((dw == 3).all())
    assert L.ef_norm_backward(ws._h, 0, 40, 0, p, 40, p, p, None, None, 0, p, 40, dw.data_ptr(), 0, None) == 0
    torch.cuda.synchronize()
    assert bool((dw == 0).all())
    args = list(backward_inputs(8, 100, torch.float32, 1))
    args[0][2, 50] = float("nan")
    dx, dw = torch.empty_like(args[0]), torch.empty(100, device="cuda")
    ef.ef_norm_backward(ws, *args, dx, dw)
    assert bool(torch.isnan(dx[2]).all()) and int(torch.isnan(dx).sum()) == 100
    assert bool(torch.isnan(dw[50])) and int(torch.isnan(dw).sum()) == 1


def test_gradient_against_differences():
    """Forward and backward pass against central differences of the forward formula in 64 bits, on rows whose normalised
    values E4M3 holds exactly: eights of numbers whose squares add up to 8."""
    rng = np.random.default_rng(5)
    eights = np.array([[2.5] + [0.5] * 7, [2, 1, 1, 1, 0.5, 0.5, 0.5, 0.5], [1.5, 1.5, 1, 1, 1, 0.5, 0.5, 0]])
    rows, n, step = 4, 72, 1e-5
    unit = np.stack([np.concatenate([rng.permutation(eights[rng.integers(3)]) for _ in range(n // 8)]) for _ in range(rows)])
    unit *= rng.choice([-1.0, 1.0], (rows, n))
    x = unit * np.array([1.0, 0.25, 8.0, 2.0])[:, None]
    w, dy, dh = (np.float64(np.float32(v)) for v in (1 + 0.3 * rng.standard_normal(n), rng.standard_normal((rows, n)), rng.standard_normal((rows, n))))

    def f(x, w):
        return float((dy * oracle.norm_forward(x, None, w, 0.0)[3]).sum() + (dh * x).sum())

    def gpu(v):
        return torch.tensor(v, dtype=torch.float32, device="cuda")

    y, act, rstd = gpu(x), checkpoint(rows, n), gpu(np.zeros(rows))
    ef.ef_norm_forward(gpu(x), None, gpu(w), 0.0, None, y, act, rstd)
    assert np.array_equal(oracle.decode(*parts(act, rows, n), n), unit)
    dx, dw = torch.empty(rows, n, device="cuda"), torch.empty(n, device="cuda")
    ef.ef_norm_backward(ef.ef_workspace_create(rows), gpu(dy), act, rstd, gpu(w), gpu(dh), dx, dw)
    # differences: a third derivative of a few tens times step^2 / 6, and 1e-16 * |f| / step
    for at in [(0, 0), (0, 9), (1, 40), (2, 63), (3, 17), (3, 71)]:
        d = np.zeros_like(x)
        d[at] = step
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * step) - f64(dx)[at]) < 2e-5
    for i in (0, 33, 71):
        d = np.zeros(n)
        d[i] = step
        assert abs((f(x, w + d) - f(x, w - d)) / (2 * step) - f64(dw)[i]) < 2e-5


def test_offsets_beyond_32_bits():
    n, stride = 1000, 1288490189
    base = torch.empty(2 * stride + n, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(base, (3, n), (stride, 1))
    x.copy_(rows_of(3, n, torch.bfloat16, 3))
    close = x.clone()
    want, got = (torch.empty(3, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a, b, rstd = checkpoint(3, n), checkpoint(3, n), torch.empty(3, device="cuda")
    ef.ef_norm_forward(close, None, None, EPS, None, want, a, rstd)
    ef.ef_norm_forward(x, None, None, EPS, None, got, b, rstd)
    assert torch.equal(want, got) and torch.equal(a, b)
    ws = ef.ef_workspace_create(3)
    ef.ef_norm_backward(ws, want, a, rstd, None, None, close, None)
    ef.ef_norm_backward(ws, want, a, rstd, None, None, x, None)
    assert torch.equal(close, x)


def test_more_rows_than_a_launch_has_threads_for():
    rows = (1 << 28) + 21            # 16 threads to a row
    x = torch.full((rows, 1), 3.0, dtype=torch.bfloat16, device="cuda")
    x[-20:, 0] = -torch.arange(1, 21, device="cuda").bfloat16()
    rstd = torch.zeros(rows, device="cuda")
    ef.ef_norm_forward(x, None, None, 0.0, None, x, None, rstd)
    assert bool((x[:-20] == 1).all()) and bool((x[-20:] == -1).all())
    assert bool(((rstd[:-20] * 3 - 1).abs() < 4 * UNIT).all())
    assert bool(((rstd[-20:] * torch.arange(1, 21, device="cuda") - 1).abs() < 4 * UNIT).all())


def test_streams_and_graphs():
    """On a stream of its own, and captured: every replay the eager result, with other work between the replays."""
    rows, n = 64, 300         # a checkpoint without padding, which no call writes
    ws = ef.ef_workspace_create(rows)
    x, w = rows_of(rows, n, torch.bfloat16, 1), torch.ones(n, device="cuda")
    y, act, rstd = torch.empty_like(x), checkpoint(rows, n), torch.empty(rows, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(n, device="cuda")

    def both():
        ef.ef_norm_forward(x, None, w, EPS, None, y, act, rstd)
        ef.ef_norm_backward(ws, y, act, rstd, w, None, dx, dw)

    both()
    want = [t.clone() for t in (y, act, dx, dw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (y, act, dx, dw):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    ef.ef_norm_forward(x, None, w, EPS, None, y, act, rstd, stream=side)
    ef.ef_norm_backward(ws, y, act, rstd, w, None, dx, dw, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, (y, act, dx, dw)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(4):
        x.copy_(rows_of(rows, n, torch.bfloat16, 10 + k))
        both()
        want = [t.clone() for t in (y, act, dx, dw)]
        for t in (y, act, dx, dw):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, act, dx, dw)))
