"""The weight gradient from a checkpoint: exactly, on whole numbers whose sums fp32 holds, and against 64 bits on others."""
import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import layer_oracle as oracle
from tests.test_act_gpu import TYPES, checkpoint, parts

pytestmark = pytest.mark.gpu

# tokens, out, width: a token and a channel; ends inside a tile, a step, a group; several tiles; many steps, cut into splits
SHAPES = [(1, 1, 1), (1, 257, 33), (15, 16, 40), (64, 256, 256), (65, 255, 257), (63, 31, 7), (129, 300, 1031), (2000, 24, 31),
          (5000, 130, 259), (700, 515, 1031), (4097, 513, 64)]
# the same for the largest tile: few steps and many, one part and several, whole rounds and a rest
LARGE = [(200, 8001, 2001), (1100, 4133, 2071), (700, 16500, 1031), (1500, 8200, 2100), (3000, 3001, 1031)]


def whole_numbers(rows, out, width, dtype, seed):
    """dz of -8..8, x of -15..15 (E4M3 holds them under any scale): sums of up to 10^5 products stay below 2^24."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randint(-15, 16, (rows, width), generator=gen).float()
    x *= (torch.rand(rows, width, generator=gen) < 0.7)
    dz = torch.randint(-8, 9, (rows, out), generator=gen).float()
    return dz, x


def encoded(x):
    act = checkpoint(*x.shape)
    ef.ef_act_encode(x.cuda(), act)
    return act


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,width", SHAPES + LARGE)
def test_whole_numbers_exactly(rows, out, width, dtype):
    dz, x = whole_numbers(rows, out, width, dtype, rows + out)
    ws = ef.ef_workspace_create(rows)
    act, z = encoded(x), dz.to(TYPES[dtype]).cuda()
    want = (dz.cuda().double().T @ x.cuda().double()).cpu()         # whole numbers, exact in any order
    flat = torch.full((out * width + 7,), 5.0, device="cuda")
    dw = flat[3:3 + out * width].view(out, width)           # 4-byte aligned, as a block of a flat gradient is
    ef.ef_weight_grad(ws, z, act, None, dw)
    assert torch.equal(dw.cpu().double(), want)
    assert bool((flat[:3] == 5).all()) and bool((flat[3 + out * width:] == 5).all())
    scale = 2.0 ** torch.randint(-3, 4, (width,), generator=torch.Generator().manual_seed(1)).float()
    ef.ef_weight_grad(ws, z, act, scale.cuda(), dw, accumulate=True)
    assert torch.equal(dw.cpu().double(), want + want * scale.double())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,width", [(333, 129, 130), (3000, 70, 300), (260, 515, 300)])
def test_against_64_bits(rows, out, width, dtype):
    gen = torch.Generator().manual_seed(rows)
    z = (torch.randn(rows, out, generator=gen) * torch.exp(2 * torch.randn(rows, 1, generator=gen))).to(TYPES[dtype])
    z[5] = 0
    x = torch.randn(rows, width, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen))
    scale = torch.randn(width, generator=gen)
    act, ws = encoded(x), ef.ef_workspace_create(rows)
    got = oracle.decode(*parts(act, rows, width), width)
    want = z.double().numpy().T @ got * scale.double().numpy()
    size = np.abs(z.double().numpy()).T @ np.abs(got) * np.abs(scale.double().numpy())
    dw = torch.empty(out, width, device="cuda")
    ef.ef_weight_grad(ws, z.cuda(), act, scale.cuda(), dw)
    # one rounding for each product added (three in fp32), at most, of a sum no larger than `size`
    off = (rows * (3 if dtype == "fp32" else 1) + 8) * oracle.EPS
    assert np.all(np.abs(dw.double().cpu().numpy() - want) <= off * size + 1e-37)
    # and as a whole: roundings of either sign
    assert np.linalg.norm(dw.double().cpu().numpy() - want) <= 4e-6 * np.linalg.norm(size)
    first = dw.clone()
    for _ in range(3):
        ef.ef_weight_grad(ws, z.cuda(), act, scale.cuda(), dw)
        assert torch.equal(dw, first)


def test_all_24_bits_of_an_fp32_gradient_count():
    gen = torch.Generator().manual_seed(2)
    z = torch.randint(-(2 ** 24) + 1, 2 ** 24, (1, 300), generator=gen).float() * 2.0 ** torch.randint(-60, 60, (1, 300), generator=gen).float()
    x = torch.zeros(1, 40)
    x[0, :] = 2.0 ** torch.arange(-3, 5).repeat(5).float()
    dw = torch.empty(300, 40, device="cuda")
    ef.ef_weight_grad(ef.ef_workspace_create(1), z.cuda(), encoded(x), None, dw)
    assert torch.equal(dw.cpu(), z.T * x)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart_at_odd_places(dtype):
    rows, out, width = 70, 131, 64
    dz, x = whole_numbers(rows, out, width, dtype, 3)
    act, want = encoded(x), dz.double().T @ x.double()
    ws = ef.ef_workspace_create(rows)
    for stride, shift in ((131, 1), (133, 0), (140, 3)):
        base = torch.full((rows * stride + 8,), float("nan"), dtype=TYPES[dtype], device="cuda")
        z = torch.as_strided(base, (rows, out), (stride, 1), shift)
        z.copy_(dz)
        dw = torch.empty(out, width, device="cuda")
        ef.ef_weight_grad(ws, z, act, None, dw)
        assert torch.equal(dw.cpu().double(), want)


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinity_stay_in_their_row_or_column(dtype):
    rows, out, width = 90, 70, 100
    dz, x = whole_numbers(rows, out, width, dtype, 8)
    want = dz.double().T @ x.double()
    dz[3, 40], dz[80, 69], x[50, 70] = float("nan"), float("inf"), float("nan")
    dw = torch.empty(out, width, device="cuda")
    ef.ef_weight_grad(ef.ef_workspace_create(rows), dz.to(TYPES[dtype]).cuda(), encoded(x), None, dw)
    dw = dw.cpu().double()
    bad = torch.zeros(out, width, dtype=torch.bool)
    bad[40], bad[69], bad[:, 64:96] = True, True, True
    assert torch.equal(dw[~bad], want[~bad])
    assert bool(torch.isnan(dw[40]).all()) and bool(torch.isnan(dw[:, 64:96]).all()) and not bool(torch.isfinite(dw[69]).any())
    nonzero = (x[80] != 0) & ~bad[0]
    assert bool(torch.isinf(dw[69][nonzero]).all())


def test_no_rows():
    L, ws = ef.lib(), ef.ef_workspace_create(4)
    some, dw = torch.zeros(64, device="cuda"), torch.full((3, 5), 2.0, device="cuda")
    for accumulate, want in ((1, 2.0), (0, 0.0)):
        assert L.ef_weight_grad(ws._h, 0, 3, 5, 1, some.data_ptr(), 3, some.data_ptr(), None, dw.data_ptr(), accumulate, None) == 0
        torch.cuda.synchronize()
        assert bool((dw == want).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("stride", [0, 1, 1 << 40])
def test_a_single_row_has_no_stride(stride, dtype):
    dz, x = whole_numbers(1, 300, 70, dtype, 4)
    z = torch.as_strided(dz.to(TYPES[dtype]).cuda(), (1, 300), (stride, 1))
    dw = torch.empty(300, 70, device="cuda")
    ef.ef_weight_grad(ef.ef_workspace_create(1), z, encoded(x), None, dw)
    assert torch.equal(dw.cpu(), dz.T * x)


def test_offsets_beyond_32_bits():
    """dz rows 1.2 * 2^30 elements apart."""
    out, width, stride = 300, 64, 1288490189
    base = torch.empty(2 * stride + out, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(base, (3, out), (stride, 1))
    dz, x = whole_numbers(3, out, width, "bf16", 4)
    z.copy_(dz)
    dw = torch.empty(out, width, device="cuda")
    ef.ef_weight_grad(ef.ef_workspace_create(3), z, encoded(x), None, dw)
    assert torch.equal(dw.cpu().double(), dz.double().T @ x.double())


def test_graph_replays():
    rows, out, width = 3000, 130, 200          # cut into splits, joined by a second kernel
    ws = ef.ef_workspace_create(rows)
    dz, x = whole_numbers(rows, out, width, "bf16", 4)
    z, act, dw = dz.bfloat16().cuda(), encoded(x), torch.empty(out, width, device="cuda")
    ef.ef_weight_grad(ws, z, act, None, dw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ef.ef_weight_grad(ws, z, act, None, dw)
    for k in range(3):
        dz = whole_numbers(rows, out, width, "bf16", 10 + k)[0]
        z.copy_(dz)
        dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw.cpu().double(), dz.double().T @ x.double())
