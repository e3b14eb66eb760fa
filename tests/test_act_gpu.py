"""Checkpoints in 8 bits, byte for byte against the definition: their arithmetic is exact but for one rounding."""
import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import layer_oracle as oracle

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def parts(act, rows, n):
    g = -(-n // 32)
    a = act.cpu().numpy()
    return a[:rows * g * 32].reshape(rows, g * 32), a[rows * g * 32:rows * g * 33].reshape(rows, g)


def checkpoint(rows, n):
    return torch.full((ef.ef_act_bytes(rows, n),), 0xA5, dtype=torch.uint8, device="cuda")


def values(rows, n, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    v = torch.randn(rows, n, generator=gen) * torch.exp(4 * torch.randn(rows, 1, generator=gen))
    v[:, ::7] *= 100.0
    v[torch.rand(rows, n, generator=gen) < 0.1] = 0.0
    return v.to(dtype)


def check(x, act, rows, n):
    codes, scales = parts(act, rows, n)
    want_codes, want_scales = oracle.encode(x.double().cpu().numpy())
    assert np.array_equal(scales, want_scales)
    same = (codes == want_codes) | (np.isnan(oracle.CODES[codes]) & np.isnan(oracle.CODES[want_codes]))
    assert same.all(), np.argwhere(~same)[:4]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (1, 32), (5, 33), (2, 1024), (67, 100), (9, 4097), (130, 259)])
def test_encode_and_decode(rows, n, dtype):
    x = values(rows, n, TYPES[dtype], 7 * rows + n).cuda()
    act = checkpoint(rows, n)
    ef.ef_act_encode(x, act)
    check(x, act, rows, n)
    codes, scales = parts(act, rows, n)
    assert not np.any(act.cpu().numpy()[codes.size + scales.size:] != 0xA5)      # what lies behind is left alone
    want = oracle.decode(codes, scales, n)
    for out in TYPES.values():
        y = torch.full((rows, n), 5.0, dtype=out, device="cuda")
        ef.ef_act_decode(act, y)
        assert np.array_equal(y.double().cpu().numpy(), want)       # bf16 holds them exactly


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_rows_apart_and_at_any_place(shift):
    rows, n, stride = 11, 77, 101
    base = values(1, rows * stride + 8, torch.bfloat16, 5).cuda()[0]
    x = torch.as_strided(base, (rows, n), (stride, 1), shift)
    act = checkpoint(rows, n)
    ef.ef_act_encode(x, act)
    check(x, act, rows, n)
    room = torch.full((rows * stride + 8,), 9.0, dtype=torch.bfloat16, device="cuda")
    y = torch.as_strided(room, (rows, n), (stride, 1), shift)
    ef.ef_act_decode(act, y)
    codes, scales = parts(act, rows, n)
    assert np.array_equal(y.double().cpu().numpy(), oracle.decode(codes, scales, n))
    kept = torch.ones_like(room, dtype=torch.bool)
    torch.as_strided(kept, (rows, n), (stride, 1), shift).fill_(False)
    assert bool((room[kept] == 9.0).all())


def test_every_size_of_scale_and_the_thresholds():
    """Largest magnitudes at 448 * 2^e and one unit above, from subnormal numbers to the largest ones."""
    tops = []
    for e in range(-140, 121):
        t = np.float64(448.0) * 2.0 ** e
        if t < 3.4e38:
            f = np.float32(t)
            tops += [f, np.nextafter(f, np.float32(np.inf)), np.nextafter(f, np.float32(0))]
    tops += [np.float32(3.4028235e38), np.float32(1e-45), np.float32(0.0), np.float32(-1e-40)]
    x = torch.zeros(len(tops), 32)
    x[:, 5] = torch.tensor(np.array(tops, np.float32))
    x[:, 6] = x[:, 5] * -0.3
    x[:, 31] = x[:, 5] * 0.0041
    x = x.cuda()
    act = checkpoint(len(tops), 32)
    ef.ef_act_encode(x, act)
    check(x, act, len(tops), 32)
    y = torch.empty_like(x)
    ef.ef_act_decode(act, y)
    assert bool(torch.isfinite(y).all())


def test_infinities_and_nan_take_their_group_and_no_other():
    for n in (32, 70, 259):
        x = values(6, n, torch.float32, n)
        x[1, 3], x[2, n - 1], x[4, n // 2] = float("inf"), float("nan"), float("-inf")
        x = x.cuda()
        act = checkpoint(6, n)
        ef.ef_act_encode(x, act)
        check(x, act, 6, n)
        y = torch.empty(6, n, device="cuda")
        ef.ef_act_decode(act, y)
        bad = torch.zeros(6, n, dtype=torch.bool)
        for r, c in ((1, 3), (2, n - 1), (4, n // 2)):
            bad[r, c // 32 * 32:c // 32 * 32 + 32] = True
        assert torch.equal(torch.isnan(y).cpu(), bad)


def test_offsets_beyond_32_bits():
    """Three rows 1.2 * 2^30 elements apart: element and byte offsets beyond 2^31 and 2^32."""
    n, stride = 1000, 1288490189
    base = torch.empty(2 * stride + n, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(base, (3, n), (stride, 1))
    x.copy_(values(3, n, torch.bfloat16, 3))
    act = checkpoint(3, n)
    ef.ef_act_encode(x, act)
    check(x, act, 3, n)
    want = x.clone()
    ef.ef_act_decode(act, want)
    x.zero_()
    ef.ef_act_decode(act, x)
    assert torch.equal(x, want)


def test_more_groups_than_a_launch_has_threads_for():
    rows = (1 << 30) + 37            # four threads to a group of one element
    x = torch.full((rows, 1), 1.0, dtype=torch.bfloat16, device="cuda")
    x[-30:, 0] = torch.arange(1, 31, device="cuda").bfloat16()
    act = torch.zeros(ef.ef_act_bytes(rows, 1), dtype=torch.uint8, device="cuda")
    ef.ef_act_encode(x, act)
    y = torch.zeros_like(x)
    ef.ef_act_decode(act, y)
    # the numbers' distance from E4M3's, which is the same under any scale
    want = x.clone()
    want[-30:] = x[-30:].float().to(torch.float8_e4m3fn).bfloat16()
    assert torch.equal(y, want)


def test_no_rows():
    x, act = torch.empty(0, 40, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    assert ef.ef_act_bytes(0, 40) == 0
    y = torch.empty(0, 40, device="cuda")
    L = ef.lib()
    some = torch.full((16,), 7, dtype=torch.uint8, device="cuda")
    assert L.ef_act_encode(0, 40, 0, some.data_ptr(), 40, some.data_ptr(), None) == 0
    assert L.ef_act_decode(0, 40, some.data_ptr(), 1, some.data_ptr(), 40, None) == 0
    assert bool((some == 7).all())
    del x, act, y
