"""Token log-probabilities and the policy loss where the logits are large numbers, finite all of them: softmax knows their differences alone."""
import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import layer_oracle as oracle
from tests.test_act_gpu import TYPES
from tests.test_policy_gpu import Case

pytestmark = pytest.mark.gpu

SIZES = [1e3, 1e6, 3e7, 1e9, 1.5e9, 3e9, 1e10, 1e12, 1e15, 1e20, 1e29, 1e31, 3e38]
# (type, vocabulary): 16, 64, 256, 512 and 1024 threads to a row, and rows read twice
TEAMS = [("bf16", 100), ("bf16", 2000), ("bf16", 9000), ("bf16", 30000), ("bf16", 50257), ("bf16", 70001), ("bf16", 196700),
         ("fp32", 100), ("fp32", 2000), ("fp32", 8000), ("fp32", 30000), ("fp32", 50257), ("fp32", 98400)]


def next_below(v):
    """The type's next number below each of v."""
    ints = torch.int16 if v.dtype is torch.bfloat16 else torch.int32
    bits = v.view(ints)
    return torch.where(v > 0, bits - 1, bits + 1).view(v.dtype)


def large_rows(vocab, dtype, extra=0):
    """For each size and sign a row of that number everywhere, one where all but a few entries are the next number below, and one that has it in one
    place among ordinary ones; `extra` ordinary rows."""
    tops = torch.tensor([s * m for m in SIZES for s in (1, -1)]).to(dtype)
    rows = 3 * len(tops) + extra
    case = Case(rows, vocab, dtype, vocab)
    for k, top in enumerate(tops):
        case.logits[3 * k] = top
        case.logits[3 * k + 1] = next_below(top[None])[0]
        case.logits[3 * k + 1, [0, vocab // 2, vocab - 1]] = top
        case.tokens[3 * k + 1] = vocab // 2
        case.logits[3 * k + 2, vocab // 3] = top
        if top > 0:
            case.tokens[3 * k + 2] = vocab // 3
    logp = torch.log_softmax(case.logits.double(), 1)[torch.arange(rows), case.tokens]
    case.old, case.ref = (logp - np.log(0.9)).float(), (logp + 0.2).float()
    case.weight[:] = 0.5
    return case


@pytest.mark.parametrize("dtype,vocab", TEAMS)
def test_large_logits(dtype, vocab):
    case = large_rows(vocab, TYPES[dtype])
    case.check(case.run())
    assert all(torch.equal(a, b) for a, b in zip(case.run(), case.run(dlogits=lambda logits: logits)))
    logp = torch.empty(len(case.tokens), device="cuda")
    ef.ef_token_logp(case.logits.cuda(), case.tokens.cuda(), logp)
    want = oracle.policy(case.logits.double().numpy(), case.tokens.numpy(), None, None, None, None, 0, 0, 0)
    assert np.all(np.abs(logp.double().cpu().numpy() - want[0]) <= want[3][0])


@pytest.mark.parametrize("dtype,vocab", [("bf16", 40000), ("bf16", 150000), ("fp32", 33000), ("fp32", 90000)])
def test_large_logits_in_slices_and_not(dtype, vocab):
    """The same rows by the kernels for few rows and by those for many."""
    many = large_rows(vocab, TYPES[dtype])
    many.check(many.run())
    few = large_rows(vocab, TYPES[dtype])
    for name in ("logits", "tokens", "old", "ref", "adv", "weight"):
        setattr(few, name, getattr(few, name)[14:78])
    few.check(few.run())
