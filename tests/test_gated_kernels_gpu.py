"""Every kernel of the gated block at sizes whose tiles it does not fill, whichever would be chosen for them, against 64 bits."""
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import train_oracle as oracle
from tests.test_gated_gpu import GATES, TYPES, blank, exact, normal, within

pytestmark = pytest.mark.gpu

# less than a step, steps and a part, many steps; tokens and channels next to the tiles' edges; rows at any place
SHAPES = [(1, 9, 3), (63, 64, 33), (65, 40, 300), (130, 129, 127), (257, 63, 129), (300, 520, 70), (513, 257, 260)]


@pytest.fixture
def kernels():
    def choose(forward=-1, backward=-1, splits=0):
        assert ef.lib().ef_gated_kernels(forward, backward, splits) == ef.EF_OK
    yield choose
    choose()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("forward", range(4))
@pytest.mark.parametrize("rows,n,f", SHAPES)
def test_forward(kind, forward, rows, n, f, kernels):
    dtype, gate, pad = TYPES[kind], "gelu" if rows % 2 else "silu", 0 if n % 8 == 0 else 3
    gen = torch.Generator("cuda").manual_seed(rows + n + f)
    x, w = normal(gen, rows, n, dtype, pad), normal(gen, 2 * f, n, dtype, pad, sigma=1.5 * n ** -0.5)
    pre, z = blank(rows, 2 * f, dtype, pad), blank(rows, f, dtype, pad)
    act, again = (torch.full((ef.ef_act_bytes(rows, f),), 9, dtype=torch.uint8, device="cuda") for _ in range(2))
    kernels(forward=forward)
    ef.ef_gated_forward(x, w, GATES[gate], pre[:, :2 * f], z[:, :f], act)
    z64, pre64, _, z_off, pre_off = oracle.gated_forward(exact(x), exact(w), gate, kind)
    within(pre[:, :2 * f], pre64, pre_off)
    within(z[:, :f], z64, z_off)
    assert bool((pre[:, 2 * f:] == 7.0).all()) and bool((z[:, f:] == 7.0).all())
    if kind == "fp32":
        ef.ef_act_encode(z[:, :f], again)
        assert torch.equal(act, again)
    # NaN in a channel's weights and in a token's input stay there, in the checkpoint's groups too, and its padding stays 0
    if f > 1:
        w[1, 0] = float("nan")
        x[0, 0] = float("inf")
        got = blank(rows, f, dtype)
        ef.ef_gated_forward(x, w, GATES[gate], None, got, act)
        assert torch.equal(got[1:, 2:], z[1:, 2:f]) and torch.equal(got[1:, :1], z[1:, :1]) and bool(torch.isnan(got[:, 1]).all())
        codes = act[:rows * ((f + 31) // 32) * 32].view(rows, -1)
        assert not codes[:, f:].any() and bool((codes[:, :min(f, 32)] == 0x7f).all())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("backward", range(4))
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("rows,n,f", SHAPES)
def test_backward(kind, backward, splits, rows, n, f, kernels):
    dtype, gate, pad = TYPES[kind], "silu" if rows % 2 else "gelu", 0 if n % 8 == 0 else 3
    gen = torch.Generator("cuda").manual_seed(rows + n * 5 + f)
    dz, pre, w = normal(gen, rows, f, dtype, pad), normal(gen, rows, 2 * f, dtype, pad, sigma=2.0), normal(gen, 2 * f, n, dtype, pad)
    ws = ef.ef_workspace_create(rows)
    dpre, dx = blank(rows, 2 * f, dtype, pad), blank(rows, n, dtype, pad)
    kernels(backward=backward, splits=splits)
    ef.ef_gated_backward(ws, dz, pre, w, GATES[gate], dpre[:, :2 * f], dx[:, :n])
    within(dpre[:, :2 * f], *oracle.gated_slopes(exact(dz), exact(pre), gate, kind))
    within(dx[:, :n], *oracle.input_grad(exact(dpre[:, :2 * f]), exact(w), kind))
    assert bool((dpre[:, 2 * f:] == 7.0).all()) and bool((dx[:, n:] == 7.0).all())


def test_other_values_are_refused():
    for args in ((4, -1, 0), (-2, -1, 0), (-1, 4, 0), (-1, -2, 0), (-1, -1, 65), (-1, -1, -1)):
        assert ef.lib().ef_gated_kernels(*args) == ef.EF_ERR_ARG
