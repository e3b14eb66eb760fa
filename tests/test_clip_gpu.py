"""Norms and clipping over many tensors, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def tensors(gen, sizes, types, sigma=1.0):
    """Tensors of their own, some of which begin in the middle of a word."""
    out = []
    for i, (n, t) in enumerate(zip(sizes, types)):
        whole = (torch.randn(n + i % 5, device="cuda", generator=gen) * sigma).to(t)
        out.append(whole[i % 5:])
    return out


def expected(grads, max_norm):
    v = np.concatenate([g.double().cpu().numpy() for g in grads]) if grads else np.zeros(0)
    norm = math.sqrt(math.fsum(v * v)) if np.isfinite(v).all() else (math.nan if np.isnan(v).any() else math.inf)
    clip = norm > max_norm and norm < math.inf
    return v, norm, max_norm / norm if clip else 1.0


def check(workers, max_norm, pad=0):
    n = sum(g.numel() for g in workers[0])
    flat, norm = torch.full((len(workers), n + pad), 7.0, device="cuda"), torch.full((len(workers),), 7.0, device="cuda")
    copies = [[g.clone() for g in w] for w in workers]
    ws = ef.ef_workspace_create(0)
    ef.ef_grad_clip(ws, workers if len(workers) > 1 else workers[0], max_norm, flat if len(workers) > 1 else flat[0], norm)
    again = torch.full_like(flat, 9.0)
    ef.ef_grad_clip(ws, workers, max_norm, again, norm.clone())
    assert torch.equal(again[:, :n].view(torch.int32), flat[:, :n].view(torch.int32))
    assert bool((flat[:, n:] == 7.0).all())
    for i, grads in enumerate(workers):
        v, want, factor = expected(grads, max_norm)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(grads, copies[i]))      # only read
        got, row = float(norm[i]), flat[i, :n].double().cpu().numpy()
        if 3.5e38 < want < math.inf:        # fp32 does not hold it: 3e38 sqrt(1033), say
            assert got == math.inf
        elif math.isfinite(want):
            assert abs(got - want) <= EPS * want * 1.001 + 2.0 ** -149
        else:
            assert got == want or (math.isnan(got) and math.isnan(want))
        if factor == 1.0:
            assert np.array_equal(row, v, equal_nan=True)
        else:
            # the factor's rounding and the product's
            assert (np.abs(row - v * factor) <= 2.01 * EPS * np.abs(v * factor) + 2.0 ** -149).all()
    # in place: rounded to the tensors' types
    ef.ef_grad_clip(ws, workers, max_norm, None, norm)
    for i, grads in enumerate(workers):
        _, _, factor = expected(copies[i], max_norm)
        for g, old in zip(grads, copies[i]):
            v = old.double().cpu().numpy() * factor
            half = (2.0 ** -8 if g.dtype == torch.bfloat16 else EPS) * 1.01
            got = g.double().cpu().numpy()
            least = 2.0 ** -133 if g.dtype == torch.bfloat16 else 2.0 ** -149
            if factor == 1.0:
                assert torch.equal(g.view(torch.uint8), old.view(torch.uint8))
            else:
                assert (np.abs(got - v) <= (half + 2.01 * EPS) * np.abs(v) + least).all()


SIZES = {"one": [1], "small": [1, 2, 3, 7, 8, 9, 64, 65], "empty between": [5, 0, 0, 3, 0], "none": [], "nothing": [0, 0], "chunk": [2048, 2047, 2049, 1, 4096, 100000],
         "many": [1 + (i * 37) % 300 for i in range(500)], "large and small": [3000001, 1, 5, 777, 1200000]}


@pytest.mark.parametrize("types", ["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("name", SIZES)
@pytest.mark.parametrize("workers", [1, 3])
def test_norm_and_clip(name, types, workers):
    sizes = SIZES[name]
    kinds = [torch.float32 if types == "fp32" or (types == "mixed" and i % 2) else torch.bfloat16 for i in range(len(sizes))]
    gen = torch.Generator("cuda").manual_seed(len(sizes))
    make = lambda: [tensors(gen, sizes, kinds, sigma=0.1 * 4 ** w) for w in range(workers)]  # noqa: E731
    for max_norm in (1.0, float(np.float32(0.01)), 1e6, 0.0, math.inf):     # the call takes a float
        check(make(), max_norm, pad=4)


def test_sizes_of_numbers():
    """Squares that fp32 does not hold, the least numbers, infinities and NaN."""
    for value in (1e30, 3e38, 1e-30, 1e-45, 0.0):
        check([[torch.full((1000,), value, device="cuda"), torch.full((33,), value, device="cuda", dtype=torch.bfloat16)]], 1.0)
        check([[torch.full((1000,), value, device="cuda")]], 2.0 ** -126)
    for bad in (math.inf, -math.inf, math.nan):
        g = [torch.randn(3000, device="cuda"), torch.randn(77, device="cuda").bfloat16()]
        g[1][5] = bad
        check([g, [t.nan_to_num(0.0, 0.0, 0.0) for t in g]], 0.5)
    # a norm beyond fp32 is infinite there, and clips by what it is
    g = torch.full((1 << 20,), 3e38, device="cuda")
    flat, norm = torch.empty(1 << 20, device="cuda"), torch.empty(1, device="cuda")
    ef.ef_grad_clip(ef.ef_workspace_create(0), [g], 1.0, flat, norm)
    assert float(norm) == math.inf and float(flat[0]) == pytest.approx(2.0 ** -10, rel=1e-6)


def test_slices_of_one_vector():
    """Blocks of a flat vector, side by side or with gaps: the same result as tensors of their own."""
    gen = torch.Generator("cuda").manual_seed(1)
    sizes = [100, 3, 5000, 1, 77]
    flat = torch.randn(2, sum(sizes) + 40, device="cuda", generator=gen)
    for gap in (0, 4, 3):
        at, parts = 0, [[], []]
        for n in sizes:
            for w in range(2):
                parts[w].append(flat[w, at:at + n])
            at += n + gap
        check([[p.clone() for p in w] for w in parts], 1.0)
        check([[p for p in w] for w in parts], 5.0)


def test_into_the_workers_step():
    """Autograd's bf16 tensors to a row of flat gradients, as the step reads it."""
    sizes = [300, 64, 1000]
    gen = torch.Generator("cuda").manual_seed(1)
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    plan, d = ef.ef_plan_create(offsets, 2), int(offsets[-1])
    workers = [tensors(gen, sizes, [torch.bfloat16, torch.float32, torch.bfloat16], sigma=2.0) for _ in range(2)]
    results = []
    for fused in (True, False):
        g, m, e = (torch.zeros(2, d, device="cuda") for _ in range(3))
        signs, scales = torch.zeros(2, plan.W, dtype=torch.int64, device="cuda"), torch.zeros(2, plan.B, device="cuda")
        norm = torch.empty(2, device="cuda")
        if fused:
            ef.ef_grad_clip(ef.ef_workspace_create(0), workers, 1.0, g, norm)
        else:
            for i, w in enumerate(workers):
                v = torch.cat([t.float() for t in w])
                g[i] = (v.double() / v.double().norm()).float()
            clean = g.clone()
        ef.ef_worker_step(plan, g, m, e, 0.9, 0.0, 0.1, signs, scales)
        results.append((signs, scales, e))
    assert torch.equal(results[0][0], results[1][0])
    # the two rows are a rounding apart at most, two half steps of an entry; so are the blocks' means of sizes, and a residual is the difference of an entry
    # (times 1 + 0.9 and the step size, rounded thrice) and its block's mean
    size = float(clean.abs().max())
    assert torch.allclose(results[0][1], results[1][1], rtol=8 * EPS) and torch.allclose(results[0][2], results[1][2], rtol=0, atol=32 * EPS * size)


def test_captured_and_replayed():
    gen = torch.Generator("cuda").manual_seed(3)
    sizes = [5000, 3, 70000]
    grads = tensors(gen, sizes, [torch.float32, torch.bfloat16, torch.float32])
    ws, flat, norm = ef.ef_workspace_create(0), torch.zeros(sum(sizes), device="cuda"), torch.zeros(1, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def step():
        ef.ef_grad_clip(ws, grads, 2.0, flat, norm)

    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    for k in range(3):
        for g in grads:
            g.normal_(generator=gen)
            g.mul_(10.0 ** (k - 2))
        step()
        want = flat.clone(), norm.clone()
        flat.zero_(), norm.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(flat, want[0]) and torch.equal(norm, want[1])
