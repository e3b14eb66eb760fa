"""Token log-probabilities and the clipped policy loss with its gradient, against 64 bits and against differences."""
import math

import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import layer_oracle as oracle
from tests.test_act_gpu import TYPES

pytestmark = pytest.mark.gpu

LOW, HIGH, KL = 0.2, 0.28, 0.05
# every team and its ends; rows held in registers, and rows read twice
VOCABS = [1, 2, 9, 259, 512, 513, 2049, 8192, 8193, 32769, 50257, 65536, 65537, 150001]


class Case:
    def __init__(self, rows, vocab, dtype, seed, pad=0, sigma=2.0):
        gen = torch.Generator().manual_seed(seed)
        live = max(1, vocab - pad)
        self.logits = torch.randn(rows, vocab, generator=gen) * sigma
        self.tokens = torch.randint(0, live, (rows,), generator=gen)
        self.logits[torch.arange(rows), self.tokens] += 5.0
        self.logits[:, live:] = -math.inf
        self.logits = self.logits.to(dtype)
        logp = torch.log_softmax(self.logits.double(), 1)[torch.arange(rows), self.tokens]
        # ratios from 0.6 to 1.7, none near the clipping's ends
        ratio = torch.tensor([0.6, 0.75, 0.9, 1.0, 1.1, 1.2, 1.35, 1.7])[torch.randint(0, 8, (rows,), generator=gen)]
        self.old = (logp - torch.log(ratio.double())).float()
        self.ref = (logp + 0.3 * torch.randn(rows, generator=gen)).float()
        self.adv = torch.randn(rows, generator=gen)
        self.weight = torch.rand(rows, generator=gen) * (torch.rand(rows, generator=gen) < 0.8)
        self.weight[0] = 0.7

    def run(self, old=True, ref=True, weight=True, dlogits=None, stream=None):
        rows, vocab = self.logits.shape
        t = {k: getattr(self, k).cuda() for k in ("logits", "tokens", "old", "ref", "adv", "weight")}
        ws = ef.ef_workspace_create(rows)
        logp, losses, loss = (torch.full((k,), 7.0, device="cuda") for k in (rows, rows, 1))
        g = torch.full_like(t["logits"], 7.0) if dlogits is None else dlogits(t["logits"])
        ef.ef_policy_loss(ws, t["logits"], t["tokens"], t["old"] if old else None, t["ref"] if ref else None, t["adv"],
                          t["weight"] if weight else None, LOW, HIGH, KL, logp, losses, loss, g, stream=stream)
        return logp, losses, loss, g

    def want(self, old=True, ref=True, weight=True):
        f = lambda k, on: getattr(self, k).double().numpy() if on else None  # noqa: E731
        return oracle.policy(f("logits", True), self.tokens.numpy(), f("old", old), f("ref", ref), f("adv", True), f("weight", weight),
                             LOW, HIGH, KL)

    def check(self, got, **kw):
        logp, losses, grad, off = self.want(**kw)
        a, b, c, d = (v.double().cpu().numpy() for v in got)
        assert np.all(np.abs(a - logp) <= off[0])
        assert np.all(np.abs(b - losses) <= off[1] + 1e-37)
        assert abs(c[0] - losses.sum()) <= off[1].sum() + 2 * oracle.EPS * abs(losses.sum()) + 1e-37
        unit = 2.0 ** -8 * (1 + 2.0 ** -7) if self.logits.dtype is torch.bfloat16 else oracle.EPS
        assert np.all(np.abs(d - grad) <= off[2] + unit * np.abs(grad))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_loss_and_gradient(vocab, dtype):
    rows = 23 if vocab < 5000 else 6
    case = Case(rows, vocab, TYPES[dtype], vocab, pad=min(7, vocab // 3))
    case.check(case.run())
    # without the old policy, the reference, the weights
    case.check(case.run(old=False), old=False)
    case.check(case.run(ref=False, weight=False), ref=False, weight=False)
    logp = torch.empty(rows, device="cuda")
    ef.ef_token_logp(case.logits.cuda(), case.tokens.cuda(), logp)
    want = oracle.policy(case.logits.double().numpy(), case.tokens.numpy(), None, None, None, None, 0, 0, 0)
    assert np.all(np.abs(logp.double().cpu().numpy() - want[0]) <= want[3][0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [33000, 41000, 50257, 57345, 70001])
def test_more_rows_of_large_vocabularies(vocab, dtype):
    """Beyond the rows that are cut into slices: a workgroup to a row, masked rows among them, also in place."""
    case = Case(66, vocab, TYPES[dtype], vocab, pad=5)
    case.tokens[3], case.logits[7] = vocab, float("nan")
    case.weight[7] = 0.0
    got = case.run()
    case.logits[7] = 0.0
    case.check(got)
    case.logits[7] = float("nan")
    assert all(torch.equal(a, b) for a, b in zip(got, case.run(dlogits=lambda logits: logits)))


@pytest.mark.parametrize("vocab,dtype", [(81921, "bf16"), (98299, "bf16"), (131073, "bf16"), (152001, "bf16"), (196601, "bf16"), (196609, "bf16"),
                                         (81923, "fp32"), (98304, "fp32"), (98305, "fp32")])
def test_the_longest_rows_in_registers(vocab, dtype):
    case = Case(65, vocab, TYPES[dtype], vocab, pad=9)
    case.weight[2], case.tokens[1] = 0.0, vocab - 10
    got = case.run()
    case.check(got)
    assert all(torch.equal(a, b) for a, b in zip(got, case.run(dlogits=lambda logits: logits)))
    logp = torch.empty(65, device="cuda")
    ef.ef_token_logp(case.logits.cuda(), case.tokens.cuda(), logp)
    live = case.weight != 0
    assert torch.equal(logp[live.cuda()], got[0][live.cuda()])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [129, 513, 767, 769, 1023, 1025, 2049, 4095, 4097, 5121, 8193, 16383, 16385, 24577, 32769, 40961, 49153, 65536])
def test_every_team(vocab, dtype):
    """Around the lengths where a row goes to another team."""
    case = Case(67, vocab, TYPES[dtype], vocab, pad=2)
    case.weight[5], case.tokens[9] = 0.0, 0
    got = case.run()
    case.check(got)
    assert all(torch.equal(a, b) for a, b in zip(got, case.run(dlogits=lambda logits: logits)))


@pytest.mark.parametrize("rows", [1, 7, 33, 64])
def test_slices(rows):
    case = Case(rows, 40001, torch.bfloat16, rows, pad=3)
    got = case.run()
    case.check(got)
    assert all(torch.equal(a, b) for a, b in zip(got, case.run(dlogits=lambda logits: logits)))


@pytest.mark.parametrize("rows", [1, 2, 255, 1030, 4000])
def test_rows(rows):
    case = Case(rows, 300, torch.bfloat16, rows)
    got = case.run()
    case.check(got)
    assert all(torch.equal(a, b) for a, b in zip(got, case.run()))      # the same bits every time


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [259, 3001, 50257, 70001])
def test_in_place_and_at_odd_places(vocab, dtype):
    case = Case(5, vocab, TYPES[dtype], 3)
    want = case.run()
    got = case.run(dlogits=lambda logits: logits)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    room = torch.full((5, vocab + 6), 4.0, dtype=TYPES[dtype], device="cuda")
    got = case.run(dlogits=lambda logits: room[:, 3:3 + vocab])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert bool((room[:, :3] == 4).all()) and bool((room[:, 3 + vocab:] == 4).all())
    wide = torch.full((5, vocab + 6), float("nan"), dtype=TYPES[dtype])
    wide[:, 1:1 + vocab] = case.logits
    logp = torch.empty(5, device="cuda")
    ef.ef_token_logp(wide.cuda()[:, 1:1 + vocab], case.tokens.cuda(), logp)
    assert torch.allclose(logp[case.weight.cuda() != 0], want[0][case.weight.cuda() != 0], rtol=0, atol=1e-6)


@pytest.mark.parametrize("vocab", [100, 1500, 9000, 50257, 70000])
def test_masked_rows_are_not_read(vocab):
    """Weight 0 or a token outside the vocabulary: whatever the logits hold."""
    case = Case(8, vocab, torch.float32, 5)
    case.weight[:] = torch.tensor([0.3, 0, 0.2, 0.1, 0.4, 0, 0.5, 0.6])
    clean = case.run()
    case.logits[1] = float("nan")
    case.logits[5] = -math.inf
    case.tokens[3], case.tokens[4], case.tokens[6] = -100, vocab, 1 << 40
    case.logits[4] = float("inf")
    logp, losses, loss, g = case.run()
    masked, kept = [1, 3, 4, 5, 6], [0, 2, 7]
    assert all(bool((v[masked] == 0).all()) for v in (logp, losses, g))
    assert all(torch.equal(v[kept], w[kept]) for v, w in zip((logp, losses, g), (clean[0], clean[1], clean[3])))
    assert abs(float(loss) - float(losses.double().sum())) <= 1e-6 * float(losses.abs().sum())
    assert not bool(torch.signbit(g[masked]).any())
    # all of them masked
    case.weight[:] = 0
    logp, losses, loss, g = case.run()
    assert all(bool((v == 0).all()) for v in (logp, losses, loss, g))
    out = torch.empty(8, device="cuda")
    case.logits[3:7] = 0.0
    ef.ef_token_logp(case.logits.cuda(), case.tokens.cuda(), out)
    assert bool((out[[3, 4, 6]] == 0).all())


@pytest.mark.parametrize("vocab", [100, 1500, 50257, 70000])
def test_infinities_and_nan(vocab):
    case = Case(7, vocab, torch.float32, 6)
    case.weight[:] = 0.5
    case.logits[1, vocab // 2] = float("nan")
    case.logits[2] = -math.inf                      # nothing is left to draw
    case.logits[3, :] = -math.inf                   # nothing but the token
    case.logits[3, case.tokens[3]] = 2.0
    case.old[3] = case.ref[3] = 0.0
    case.logits[4, 7] = float("inf")
    case.logits[5] = torch.finfo(torch.float32).min     # a mask of the lowest value
    case.logits[5, case.tokens[5]] = 1.0
    case.old[5] = case.ref[5] = 0.0
    case.logits[6] = torch.finfo(torch.float32).min     # in every place: all alike
    case.old[6] = case.ref[6] = -math.log(vocab)
    logp, losses, _, g = case.run()
    assert all(bool(torch.isnan(v[1]).any()) for v in (logp, losses)) and bool(torch.isnan(g[1]).all())
    assert bool(torch.isnan(logp[2])) and bool(torch.isnan(g[2]).all())
    assert bool(torch.isnan(logp[4])) or float(logp[4]) == -math.inf
    for t in (3, 5):
        assert float(logp[t]) == 0.0
        assert float(g[t].abs().max()) <= 1e-6 * abs(0.5 * float(case.adv[t]))
    assert abs(float(logp[6]) + math.log(vocab)) < 1e-5
    fine = [0]
    want = case.want()
    assert np.all(np.abs(g.double().cpu().numpy()[fine] - want[2][fine]) <= want[3][2][fine] + oracle.EPS * np.abs(want[2][fine]))


def test_the_tokens_own_logit_ruled_out():
    """-inf at the token itself: its probability is 0, the ratio 0."""
    case = Case(2, 400, torch.float32, 8)
    case.logits[0, case.tokens[0]] = -math.inf
    case.adv[0] = 1.0
    logp, losses, _, g = case.run(ref=False)
    assert float(logp[0]) == -math.inf and float(losses[0]) == 0.0 and bool((g[0] == 0).all())


def test_forward_alone_and_large_values():
    case = Case(9, 1000, torch.float32, 11, sigma=30.0)
    logp, losses, loss, g = case.run()
    case.check((logp, losses, loss, g))
    ws = ef.ef_workspace_create(9)
    only = torch.empty(1, device="cuda")
    ef.ef_policy_loss(ws, case.logits.cuda(), case.tokens.cuda(), case.old.cuda(), case.ref.cuda(), case.adv.cuda(), case.weight.cuda(),
                      LOW, HIGH, KL, None, None, only, None)
    assert torch.equal(only, loss)
    shifted = case.logits + 4096.0          # softmax does not see it; the logits lose bits
    out = torch.empty(9, device="cuda")
    ef.ef_token_logp(shifted.cuda(), case.tokens.cuda(), out)
    want = torch.log_softmax(shifted.double(), 1)[torch.arange(9), case.tokens]
    assert float((out.cpu().double() - want).abs().max()) < 1e-4


def test_clipping_takes_the_gradient_where_it_should():
    """Above 1 + high with a positive advantage, below 1 - low with a negative one: no gradient; else the ratio's."""
    ratios, advs = [0.5, 0.5, 1.0, 1.0, 2.0, 2.0], [1.0, -1.0, 1.0, -1.0, 1.0, -1.0]
    logits = torch.randn(6, 50, generator=torch.Generator().manual_seed(1))
    tokens = torch.arange(6)
    logp = torch.log_softmax(logits.double(), 1)[torch.arange(6), tokens]
    case = Case(6, 50, torch.float32, 1)
    case.logits, case.tokens, case.adv = logits, tokens, torch.tensor(advs)
    case.old, case.weight = (logp - torch.log(torch.tensor(ratios).double())).float(), torch.ones(6)
    _, losses, _, g = case.run(ref=False)
    moved = g.abs().amax(1).cpu() > 0
    assert moved.tolist() == [True, False, True, True, False, True]
    want = [-0.5, 0.8, -1.0, 1.0, -1.28, 2.0]
    assert np.allclose(losses.cpu().numpy(), want, rtol=0, atol=1e-5)


def test_gradient_against_differences():
    case = Case(4, 40, torch.float32, 12)
    case.weight[:] = torch.tensor([0.5, 1.0, 0.25, 2.0])
    g = case.run()[3].double().cpu().numpy()

    def f(logits):
        return oracle.policy(logits, case.tokens.numpy(), case.old.double().numpy(), case.ref.double().numpy(), case.adv.double().numpy(),
                             case.weight.double().numpy(), LOW, HIGH, KL)[1].sum()

    x, step = case.logits.double().numpy(), 1e-5
    for at in [(t, v) for t in range(4) for v in (0, 17, 39, int(case.tokens[t]))]:
        d = np.zeros_like(x)
        d[at] = step
        assert abs((f(x + d) - f(x - d)) / (2 * step) - g[at]) < 2e-6


def test_offsets_beyond_32_bits():
    vocab, stride = 50257, 1288490189
    case = Case(3, vocab, torch.bfloat16, 13)
    want = case.run()
    base = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(base, (3, vocab), (stride, 1))
    got = case.run(dlogits=lambda logits: rows)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    rows.copy_(case.logits)
    logp = torch.empty(3, device="cuda")
    ef.ef_token_logp(rows, case.tokens.cuda(), logp)
    live = case.weight != 0
    assert torch.equal(logp[live.cuda()], want[0][live.cuda()])


@pytest.mark.parametrize("shift", [0, 1, 5])
def test_the_largest_vocabulary(shift):
    vocab = (1 << 31) - 1
    base = torch.zeros(vocab + 16, dtype=torch.bfloat16, device="cuda")
    row = base[shift:shift + vocab].view(1, vocab)
    tokens, one = torch.tensor([vocab - 1], device="cuda"), torch.ones(1, device="cuda")
    logp, losses, loss = (torch.empty(1, device="cuda") for _ in range(3))
    ef.ef_policy_loss(ef.ef_workspace_create(1), row, tokens, None, None, one, None, 0.2, 0.2, 0.0, logp, losses, loss, row)
    # equal logits: every sum of exponentials is a whole number that fp32 holds or is next to
    assert abs(float(logp) + 31 * np.log(2)) < 4e-6 and float(loss) == -1.0
    p = torch.tensor(2.0 ** -31).bfloat16()
    assert bool((row[0, :-1] == p.cuda()).all()) and float(row[0, -1]) == -1.0
    assert bool((base[:shift] == 0).all()) and bool((base[shift + vocab:] == 0).all())


def test_streams_and_graphs():
    case = Case(40, 600, torch.bfloat16, 14)
    want = case.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    t = {k: getattr(case, k).cuda() for k in ("logits", "tokens", "old", "ref", "adv", "weight")}
    ws = ef.ef_workspace_create(40)
    out = [torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros_like(t["logits"])]

    def call(stream=None):
        ef.ef_policy_loss(ws, t["logits"], t["tokens"], t["old"], t["ref"], t["adv"], t["weight"], LOW, HIGH, KL, *out, stream=stream)

    side.wait_stream(torch.cuda.current_stream())
    call(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        t["logits"].copy_(Case(40, 600, torch.bfloat16, 20 + k).logits)
        call()
        want = [v.clone() for v in out]
        for v in out:
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
