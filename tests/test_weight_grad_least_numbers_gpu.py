"""Gradients next to the types' least numbers in the weight gradient: bf16 counts whole, fp32 down to bf16's least number, 2^-133."""
import pytest
import torch

import paper_1905_10936_amd as ef
from tests.test_weight_grad_gpu import encoded

pytestmark = pytest.mark.gpu


def weight_grad(z, power, out, width=40):
    """dw for one token of gradient z and inputs of 2^power."""
    dw = torch.empty(out, width, device="cuda")
    ef.ef_weight_grad(ef.ef_workspace_create(1), z.cuda(), encoded(torch.full((1, width), 2.0 ** power)), None, dw)
    return dw.cpu().double()


@pytest.mark.parametrize("out", [70, 300])
def test_bf16(out):
    z = (torch.randint(-255, 256, (1, out), generator=torch.Generator().manual_seed(out)).double() * 2.0 ** -133).bfloat16()
    for power in (0, 60):
        assert torch.equal(weight_grad(z, power, out), (z.double().T * 2.0 ** power).expand(out, 40))


@pytest.mark.parametrize("out", [70, 300])
def test_fp32(out):
    whole = torch.randint(-(2 ** 24) + 1, 2 ** 24, (1, out), generator=torch.Generator().manual_seed(out))
    z = (whole.double() * 2.0 ** -149).float()
    assert torch.equal(z.double() * 2.0 ** 149, whole.double())
    kept = torch.trunc(whole.double() * 2.0 ** -16) * 2.0 ** -133
    assert torch.equal(weight_grad(z, 60, out), (kept.T * 2.0 ** 60).expand(out, 40))
