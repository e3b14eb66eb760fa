"""The native marshalling of the layers' calls (csrc/ef_binding.cpp) against the path through ctypes: the same bits for every form of their
arguments, and the same exceptions for what neither takes."""
import pytest
import torch

import paper_1905_10936_amd as ef

pytestmark = pytest.mark.gpu


class _Recorder:
    """A native module, and which of its calls answered."""

    def __init__(self, native):
        self.native, self.answers = native, []

    def __getattr__(self, name):
        def call(*args):
            rc = getattr(self.native, name)(*args)
            self.answers.append((name, rc is not None))
            return rc
        return call


def _run(dtype, rows, n, pad, bare):
    gen = torch.Generator("cuda").manual_seed(rows * n + pad)

    def matrix(width=n):
        t = torch.randn(rows, width + pad, device="cuda", generator=gen).to(dtype)[:, :width]
        return t[0] if rows == 1 and pad == 0 else t

    ws, v = ef.ef_workspace_create(rows), lambda k: torch.zeros(k, device="cuda")  # noqa: E731
    x, r, h, y, dx = matrix(), matrix(), matrix(), matrix(), matrix()
    act, act2 = (torch.zeros(ef.ef_act_bytes(rows, n), dtype=torch.uint8, device="cuda") for _ in range(2))
    w, rstd, dw = 1 + torch.rand(n, device="cuda", generator=gen), v(rows), v(n)
    ef.ef_norm_forward(x, None if bare else r, None if bare else w, 1e-5, None if bare else h, y, act, rstd)
    ef.ef_norm_backward(ws, y, act, rstd, None if bare else w, None if bare else h, dx, None if bare else dw, accumulate=not bare)
    ef.ef_act_encode(x, act2)
    ef.ef_act_decode(act2, r)
    out = v(11 * n).view(11, n)
    ef.ef_weight_grad(ws, matrix(11), act, None if bare else w, out, True)
    tokens = torch.arange(rows, device="cuda") % n
    logp, losses, loss, extra = v(rows), v(rows), v(1), v(rows)
    ef.ef_token_logp(x, tokens, extra)
    old, adv = extra - 0.1, torch.randn(rows, device="cuda", generator=gen)
    ef.ef_policy_loss(ws, x, tokens, None if bare else old, None if bare else extra, adv, None if bare else adv.abs(), 0.2, 0.3, 0.1, logp,
                      None if bare else losses, loss, None if bare else h)
    return [t.clone() for t in (h, y, dx, act, act2, rstd, dw, r, out, logp, losses, loss, extra)]


@pytest.mark.parametrize("bare", [False, True])
@pytest.mark.parametrize("dtype,rows,n,pad", [(torch.bfloat16, 7, 100, 0), (torch.float32, 1, 33, 0), (torch.bfloat16, 5, 64, 3), (torch.float32, 40, 700, 9)])
def test_same_bits(dtype, rows, n, pad, bare, monkeypatch):
    ef.lib()                # which loads the native calls
    recorder = _Recorder(ef._native)
    monkeypatch.setattr(ef, "_native", recorder)
    native = _run(dtype, rows, n, pad, bare)
    assert len(recorder.answers) == 7 and all(answered for _, answered in recorder.answers), recorder.answers
    monkeypatch.setattr(ef, "_native", ef._ThroughCtypes())
    for a, b in zip(native, _run(dtype, rows, n, pad, bare)):
        assert torch.equal(a, b)


def test_refusals_through_either():
    ws = ef.ef_workspace_create(4)
    x, act, v = torch.zeros(4, 64, device="cuda"), torch.zeros(ef.ef_act_bytes(4, 64), dtype=torch.uint8, device="cuda"), torch.zeros(4, device="cuda")
    tokens, g = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, 64, device="cuda")
    for call, error in (
            (lambda: ef.ef_act_encode(x, act[:-1]), TypeError), (lambda: ef.ef_act_encode(x.half(), act), TypeError),
            (lambda: ef.ef_act_encode(x.t(), act), TypeError), (lambda: ef.ef_act_encode(x.cpu(), act), TypeError),
            (lambda: ef.ef_act_decode(act, x.double()), TypeError),
            (lambda: ef.ef_norm_forward(x, x[:3], None, 1e-6, None, g, None, None), TypeError),
            (lambda: ef.ef_norm_forward(x, x.bfloat16(), None, 1e-6, None, g, None, None), TypeError),
            (lambda: ef.ef_norm_forward(x, None, v, 1e-6, None, g, None, None), TypeError),
            (lambda: ef.ef_norm_forward(x, None, None, 1e-6, None, None, None, None), ef.EfError),
            (lambda: ef.ef_norm_forward(x, None, None, -1.0, None, g, None, None), ef.EfError),
            (lambda: ef.ef_norm_forward(x, None, None, 1e-6, None, x[:, 1:], None, None), TypeError),
            (lambda: ef.ef_norm_backward(ws, x, act, v[:3], None, None, g, None), TypeError),
            (lambda: ef.ef_norm_backward(ws, x, act, v, None, None, None, None), ef.EfError),
            (lambda: ef.ef_norm_backward(None, x, act, v, None, None, g, None), TypeError),
            (lambda: ef.ef_weight_grad(ws, g[:, :3], act, None, g[:3].t()), TypeError),
            (lambda: ef.ef_weight_grad(ws, g[:, :3], act, None, g[:2]), TypeError),
            (lambda: ef.ef_token_logp(x, tokens.int(), v), TypeError), (lambda: ef.ef_token_logp(x, tokens, v.double()), TypeError),
            (lambda: ef.ef_policy_loss(ws, x, tokens, v, v, None, v, 0.2, 0.2, 0.0, None, None, None, g), ef.EfError),
            (lambda: ef.ef_policy_loss(ws, x, tokens, v, v, v, v, 0.2, 0.2, 0.0, None, None, None, None), ef.EfError),
            (lambda: ef.ef_policy_loss(ws, torch.zeros(5, 64, device="cuda"), tokens.new_zeros(5), None, None, torch.zeros(5, device="cuda"), None, 0.2,
                                       0.2, 0.0, None, None, torch.zeros(1, device="cuda"), None), ef.EfError)):
        with pytest.raises(error):
            call()
    ws.close()
    with pytest.raises(ef.EfError) as e:
        ef.ef_norm_backward(ws, x, act, v, None, None, g, None)
    assert e.value.code == ef.EF_ERR_NULL
