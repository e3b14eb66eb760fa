"""The gated block on rows so far apart that 32 bits do not hold the way from one to another, or just hold it: as from rows one behind the other, bit for bit."""
import pytest
import torch

import paper_1905_10936_amd as ef
from tests.test_gated_gpu import GATES, TYPES, blank, normal
from tests.test_gated_kernels_gpu import kernels  # noqa: F401

pytestmark = pytest.mark.gpu

SIZE = {"bf16": 2, "fp32": 4}


def apart(t, stride):
    """The same rows, `stride` elements apart."""
    far = torch.empty((t.shape[0] - 1) * stride + t.shape[1], device="cuda", dtype=t.dtype).as_strided(t.shape, (stride, 1))
    far.copy_(t)
    return far


def reach(kind, rows):
    """The largest stride at which `rows` rows and one more are within 32 bits of one another."""
    return (1 << 32) // SIZE[kind] // (rows + 1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("forward,tokens,channels", [(0, 32, 16), (1, 256, 128), (2, 128, 64), (3, 64, 64)])
def test_forward(kind, forward, tokens, channels, kernels):  # noqa: F811
    """x, then w, at the last stride whose offsets the kernel keeps in 32 bits, and beyond it."""
    dtype, rows, n, f = TYPES[kind], 70, 150, 6
    gen = torch.Generator("cuda").manual_seed(forward)
    x, w = normal(gen, rows, n, dtype), normal(gen, 2 * f, n, dtype, sigma=0.1)
    kernels(forward=forward)
    want = [blank(rows, 2 * f, dtype), blank(rows, f, dtype), torch.zeros(ef.ef_act_bytes(rows, f), dtype=torch.uint8, device="cuda")]
    ef.ef_gated_forward(x, w, GATES["silu"], *want)
    for x_stride, w_stride in ((reach(kind, tokens), n), (reach(kind, tokens) + 3, n), (n, reach(kind, f + channels)), (n, reach(kind, f + channels) + 1)):
        got = [torch.zeros_like(t) for t in want]
        ef.ef_gated_forward(apart(x, x_stride), apart(w, w_stride), GATES["silu"], *got)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (x_stride, w_stride)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("backward,tokens", [(0, 256), (1, 128), (2, 128), (3, 64)])
@pytest.mark.parametrize("splits", [1, 2])
def test_backward(kind, backward, tokens, splits, kernels):  # noqa: F811
    """dpre, then w, likewise; the other matrices as far apart as dpre."""
    dtype, rows, n, f = TYPES[kind], 20, 90, 70
    gen = torch.Generator("cuda").manual_seed(backward)
    dz, pre, w = normal(gen, rows, f, dtype), normal(gen, rows, 2 * f, dtype, sigma=2.0), normal(gen, 2 * f, n, dtype)
    ws = ef.ef_workspace_create(rows)
    kernels(backward=backward, splits=splits)
    want = blank(rows, 2 * f, dtype), blank(rows, n, dtype)
    ef.ef_gated_backward(ws, dz, pre, w, GATES["gelu"], *want)
    for stride, w_stride in ((reach(kind, tokens), n), (reach(kind, tokens) + 1, n), (2 * f, 1 << 24), (2 * f, (1 << 24) + 1)):
        got = apart(torch.zeros_like(want[0]), stride), apart(torch.zeros_like(want[1]), max(stride, n))
        ef.ef_gated_backward(ws, apart(dz, stride), apart(pre, stride), apart(w, w_stride), GATES["gelu"], *got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (stride, w_stride)
        del got


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("forward", range(4))
def test_results_far_apart(kind, forward, kernels):  # noqa: F811
    """Rows of z and pre more than 4 GB from the first."""
    dtype, rows, n, f, stride = TYPES[kind], 6, 40, 33, (1 << 29) + 3
    gen = torch.Generator("cuda").manual_seed(9)
    x, w = normal(gen, rows, n, dtype), normal(gen, 2 * f, n, dtype, sigma=0.2)
    kernels(forward=forward)
    want = blank(rows, 2 * f, dtype), blank(rows, f, dtype)
    ef.ef_gated_forward(x, w, GATES["gelu"], *want, None)
    got = torch.empty(5 * stride + 3 * f, device="cuda", dtype=dtype).as_strided((rows, 3 * f), (stride, 1))
    ef.ef_gated_forward(x, w, GATES["gelu"], got[:, :2 * f], got[:, 2 * f:], None)
    assert torch.equal(got[:, :2 * f], want[0]) and torch.equal(got[:, 2 * f:], want[1])
