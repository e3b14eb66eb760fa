"""Calls without rows through the Python binding, with empty tensors, whose address is null: sums over nothing are zero, or what was there."""
import pytest
import torch

import paper_1905_10936_amd as ef

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "ctypes"])
def binding(request, monkeypatch):
    ef.lib()
    if request.param == "ctypes":
        monkeypatch.setattr(ef, "_native", ef._ThroughCtypes())


def nothing(*shape, dtype=torch.float32):
    t = torch.empty(0, *shape, dtype=dtype, device="cuda")
    assert t.data_ptr() == 0
    return t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_call(dtype, binding):
    n, out = 40, 7
    ws = ef.ef_workspace_create(5)
    x, act, rows, tokens = nothing(n, dtype=dtype), nothing(dtype=torch.uint8), nothing(), nothing(dtype=torch.int64)
    w = torch.ones(n, device="cuda")
    ef.ef_act_encode(x, act)
    ef.ef_act_decode(act, x)
    ef.ef_norm_forward(x, x.clone(), w, 1e-6, x.clone(), x.clone(), act, rows)
    ef.ef_norm_forward(x, None, None, 1e-6, None, None, None, rows)
    ef.ef_token_logp(x, tokens, rows)
    for accumulate, want in ((True, 3.0), (False, 0.0)):
        dweight, dw = torch.full((n,), 3.0, device="cuda"), torch.full((out, n), 3.0, device="cuda")
        ef.ef_norm_backward(ws, x, act, rows, w, x.clone(), x.clone(), dweight, accumulate)
        assert bool((dweight == want).all())
        ef.ef_weight_grad(ws, nothing(out, dtype=dtype), act, w, dw, accumulate)
        assert bool((dw == want).all())
    ef.ef_norm_backward(ws, x, act, rows, None, None, x.clone(), None)
    loss = torch.full((1,), 3.0, device="cuda")
    ef.ef_policy_loss(ws, x, tokens, rows, rows.clone(), rows.clone(), rows.clone(), 0.2, 0.2, 0.1, rows.clone(), rows.clone(), loss, x)
    assert float(loss) == 0.0
    ef.ef_policy_loss(ws, x, tokens, None, None, rows, None, 0.2, 0.2, 0.0, None, None, None, x.clone())


def test_what_is_missing_is_missing_without_rows_too(binding):
    ws, x, act, rows, tokens = ef.ef_workspace_create(5), nothing(40), nothing(dtype=torch.uint8), nothing(), nothing(dtype=torch.int64)
    for call in (lambda: ef.ef_act_encode(x, None), lambda: ef.ef_act_decode(None, x),
                 lambda: ef.ef_norm_forward(x, x.clone(), None, 1e-6, None, None, None, None),
                 lambda: ef.ef_norm_backward(ws, x, None, rows, None, None, x.clone(), None),
                 lambda: ef.ef_norm_backward(ws, x, act, None, None, None, x.clone(), None),
                 lambda: ef.ef_norm_backward(ws, x, act, rows, None, None, None, torch.zeros(40, device="cuda")),
                 lambda: ef.ef_weight_grad(ws, x, None, None, torch.zeros(40, 8, device="cuda")),
                 lambda: ef.ef_token_logp(x, None, rows), lambda: ef.ef_token_logp(x, tokens, None),
                 lambda: ef.ef_policy_loss(ws, x, tokens, None, None, None, None, 0.2, 0.2, 0.0, rows, None, None, None),
                 lambda: ef.ef_policy_loss(ws, x, None, None, None, rows, None, 0.2, 0.2, 0.0, rows.clone(), None, None, None),
                 lambda: ef.ef_policy_loss(ws, x, tokens, None, None, rows, None, 0.2, 0.2, 0.0, None, None, None, None)):
        with pytest.raises(ef.EfError) as e:
            call()
        assert e.value.code == ef.EF_ERR_NULL
