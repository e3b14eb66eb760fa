"""The gate's activations at every size, in both types and in every kernel, against 64 bits: sigmoids that end, activations next to the type's largest, infinities, NaN."""
import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import train_oracle as oracle
from tests.test_gated_gpu import GATES, TYPES, blank, exact
from tests.test_gated_kernels_gpu import kernels  # noqa: F401

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -126     # a sigmoid below it may be 0, and so may a result
A = sorted({s * v for s in (1, -1) for v in (0, 1e-40, 1e-20, 1e-3, 0.5, 1, 2, 3, 5, 7, 8, 9, 9.5, 9.75, 10, 10.25, 12, 15, 16.5, 40, 70, 80, 84, 86, 87, 87.5, 88, 88.5, 89, 90, 95,
                                               100, 104, 110, 1e4, 1e18, 1e30, 3e38)})
U = (1.0, -2.5, 1e-30, 1e30)


def inputs(dtype):
    a, u = torch.tensor([(a, u) for a in A for u in U if abs(a) * abs(u) < 3.2e38 or u == 1.0], device="cuda").to(dtype).unbind(1)
    return a, u


def error(s):
    """Relative error of an activation in fp32: F's constants and roundings, 6 half steps of it, the exponent's two, the exponential, the sum, the reciprocal and two products."""
    return (np.minimum(np.abs(s), 200.0) * 8 + 8) * oracle.EPS


def agree(got, want, off, kind, a, u):
    got = exact(got)
    limit = float(torch.finfo(TYPES[kind]).max)
    off = off + (np.abs(want) + off) * oracle.HALF_STEP[kind] + LEAST
    bad = ~((np.abs(got - want) <= off) | ((np.abs(want) + off > limit) & (got == np.copysign(np.inf, want))))
    assert not bad.any(), (a[bad][:4], u[bad][:4], got[bad][:4], want[bad][:4], off[bad][:4])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("forward", range(4))
def test_forward(kind, gate, forward, kernels):  # noqa: F811
    a, u = inputs(TYPES[kind])
    rows = a.numel()
    z, pre = blank(rows, 1, TYPES[kind]), blank(rows, 2, TYPES[kind])
    kernels(forward=forward)
    ef.ef_gated_forward(torch.stack([a, u], 1), torch.eye(2, device="cuda", dtype=TYPES[kind]), GATES[gate], pre, z, None)
    assert torch.equal(pre, torch.stack([a, u], 1))
    a, u = exact(a), exact(u)
    s, _ = oracle.inner_slope(a, gate)
    act, _, _ = oracle.activation(a, gate)
    agree(z[:, 0], act * u, np.abs(act * u) * error(s) + np.abs(a * u) * LEAST, kind, a, u)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gate", GATES)
def test_backward(kind, gate):
    a, u = inputs(TYPES[kind])
    rows = a.numel()
    dz, dpre, ws = torch.full((rows, 1), 0.5, device="cuda", dtype=TYPES[kind]), blank(rows, 2, TYPES[kind]), ef.ef_workspace_create(rows)
    ef.ef_gated_backward(ws, dz, torch.stack([a, u], 1), torch.eye(2, device="cuda", dtype=TYPES[kind]), GATES[gate], dpre, None)
    a, u = exact(a), exact(u)
    s, ds = oracle.inner_slope(a, gate)
    act, slope, _ = oracle.activation(a, gate)
    with np.errstate(over="ignore"):
        small = np.exp(-np.abs(s))
    sig, both = np.where(s < 0, small, 1.0) / (1 + small), small / (1 + small) ** 2
    # act' is a sum of two parts, of which each has its error, and either sigmoid may be 0 below LEAST: then so is the second part
    size = sig + np.abs(a) * both * ds
    ended = np.where(both < 2 * LEAST, 2 * LEAST + np.abs(a) * both * ds, LEAST)
    agree(dpre[:, 0], 0.5 * u * slope, 0.5 * np.abs(u) * (size * 2 * error(s) + ended), kind, a, u)
    agree(dpre[:, 1], 0.5 * act, 0.5 * (np.abs(act) * error(s) + np.abs(a) * LEAST), kind, a, u)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("forward", range(4))
def test_infinities_and_nan(kind, gate, forward, kernels):  # noqa: F811
    """As the formula has them: -inf times a sigmoid of 0 is a NaN."""
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([inf, -inf, nan, 1.0], device="cuda", dtype=TYPES[kind])[:, None]
    z, dpre, ws = blank(4, 1, TYPES[kind]), blank(4, 2, TYPES[kind]), ef.ef_workspace_create(4)
    kernels(forward=forward)
    ef.ef_gated_forward(x, torch.ones(2, 1, device="cuda", dtype=TYPES[kind]), GATES[gate], None, z, None)
    assert z[0] == inf and torch.isnan(z[1:3]).all() and torch.isfinite(z[3])
    ef.ef_gated_backward(ws, torch.ones_like(x), torch.cat([x, torch.ones_like(x)], 1), torch.ones(2, 1, device="cuda", dtype=TYPES[kind]), GATES[gate], dpre, None)
    assert dpre[0].tolist() == [1.0, inf] and dpre[1, 0] == 0 and torch.isnan(dpre[1, 1]) and torch.isnan(dpre[2]).all() and torch.isfinite(dpre[3]).all()
