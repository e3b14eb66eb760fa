"""RMS norm of rows whose squares fp32 does not hold: the normalised row is of ordinary size whatever the row's."""
import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests.test_act_gpu import TYPES, checkpoint
from tests.test_norm_gpu import UNIT, check_forward, f64, rows_of

pytestmark = pytest.mark.gpu

# every team
WIDTHS = [1, 100, 128, 500, 1024, 1500, 2048, 4096, 6000, 8200, 16384]
SCALES = [1e-40, 1e-38, 1e-33, 1e-27, 1e-24, 1e-22, 1e-21, 1e-19, 1e-15, 1.0, 1e15, 1e17, 1e18, 1e19, 1e20, 1e25, 1e30, 1e34, 1e36]


def check(x, residual, weight, eps):
    rows, n = x.shape
    h, y, rstd, act = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), checkpoint(rows, n)
    ef.ef_norm_forward(x, residual, weight, eps, h, y, act, rstd)
    v = f64(x) if residual is None else f64(x) + f64(residual)
    want = 1.0 / np.sqrt((v * v).mean(1) + float(np.float32(eps)))
    got = f64(rstd)
    fits = want < 3.4e38            # beyond fp32 it is infinite; below its normal numbers it is off by half the least one
    assert np.all(np.abs(got - want)[fits] <= (30 * UNIT * want + 2.0 ** -150)[fits]) and np.all(np.isinf(got[~fits]))
    check_forward(x, residual, weight, h, y, act, torch.from_numpy(want), float(np.float32(eps)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", WIDTHS)
def test_large_and_small_rows(n, dtype):
    scale = torch.tensor(SCALES, dtype=torch.float64)[:, None]
    rows = len(SCALES)

    def make(seed):
        v = rows_of(rows, n, torch.float32, seed).cpu().double() * scale
        return v.to(TYPES[dtype]).cuda()

    x, r, w = make(n), make(n + 1), 1 + 0.2 * torch.rand(n, device="cuda")
    x[:, 0] = (scale[:, 0] * 3).to(TYPES[dtype]).cuda()             # no row of zeros
    r[:, 0] = x[:, 0]
    for eps in (0.0, 1e-44, 1e-30, 1e-12, 1e-6, 1.0):
        check(x, None, None, eps)
        check(x, r, w, eps)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_largest_and_the_least(dtype):
    t = TYPES[dtype]
    least = 2.0 ** -133 if t is torch.bfloat16 else 2.0 ** -149
    for n in (7, 1024, 3000, 9000):
        x = torch.empty(4, n, dtype=t, device="cuda")
        x[0], x[1], x[2] = torch.finfo(t).max, torch.finfo(t).min, least
        x[3], x[3, ::2] = torch.finfo(t).max, 1.0
        check(x, None, None, 0.0)
        check(x[[0, 1, 3]].contiguous(), None, None, 1e38)


def test_many_ordinary_and_few_large_rows():
    """Rows of either kind in one wavefront and one workgroup; ordinary rows are what they are alone."""
    for n in (60, 700, 5000):
        x = rows_of(50, n, torch.float32, n)
        y, again = torch.empty_like(x), torch.empty_like(x)
        ef.ef_norm_forward(x, None, None, 1e-6, None, y, None, None)
        other = x.clone()
        other[::3] *= 1e25
        ef.ef_norm_forward(other, None, None, 1e-6, None, again, None, None)
        keep = torch.ones(50, dtype=torch.bool)
        keep[::3] = False
        assert torch.equal(y[keep.cuda()], again[keep.cuda()])
        check(other, None, None, 1e-6)
