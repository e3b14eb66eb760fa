"""Drawing tokens, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_1905_10936_amd as ef
from tests import train_oracle as oracle

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SETTINGS = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}


def draw(logits, uniform, logp=True, ws=None, **settings):
    rows = logits.shape[0]
    tokens = torch.full((rows,), -7, dtype=torch.int64, device="cuda")
    out = torch.full((rows,), 7.0, device="cuda") if logp else None
    ef.ef_sample_tokens(ws or ef.ef_workspace_create(rows), logits, uniform, *(settings.get(k) for k in SETTINGS), tokens, out)
    return tokens, out


def check(logits, uniform, **settings):
    tokens, logp = draw(logits, uniform, **settings)
    v, u = logits.double().cpu().numpy(), uniform.double().cpu().numpy()
    s = {k: t.double().cpu().numpy() for k, t in settings.items()}
    got, got_logp = tokens.tolist(), logp.double().tolist()
    for i in range(len(v)):
        right, want = oracle.sample(v[i], u[i], *(s[k][i] if k in s else other for k, other in zip(SETTINGS, (1.0, 0, 1.0, 0.0))))
        assert got[i] in right, (i, got[i], right, {k: t[i] for k, t in s.items()}, u[i])
        if got[i] < 0:
            assert math.isnan(got_logp[i])
        else:
            # one rounding of the result; the sum's exponentials are fp32's: x = v - top, its product with log2(e) and that factor are rounded, 2.3 |x| half
            # steps of a term in all, the exponential by 2, sums of eight by 3; the mean of |x| over the distribution is its entropy less the sum's
            # logarithm, at most log(n)
            off = 2.0 ** -24 * (abs(want[got[i]]) + 2.3 * math.log(v.shape[1]) + 5) + 1e-9
            assert abs(got_logp[i] - want[got[i]]) <= off, i
    again, _ = draw(logits, uniform, logp=False, **settings)
    assert torch.equal(tokens, again)
    return tokens


def column(rows, value, kind):
    return torch.full((rows,), value, device="cuda", dtype=SETTINGS[kind])


def mixed(rows, gen, vocab):
    r = lambda: torch.rand(rows, device="cuda", generator=gen)  # noqa: E731
    return {"temperature": torch.where(r() < 0.15, torch.zeros(rows, device="cuda"), 0.3 + 1.5 * r()),
            "top_k": torch.where(r() < 0.3, torch.zeros(rows, device="cuda"), torch.exp(r() * math.log(2.0 * vocab + 1))).to(torch.int32),
            "top_p": torch.where(r() < 0.3, torch.ones(rows, device="cuda"), r()), "min_p": torch.where(r() < 0.5, torch.zeros(rows, device="cuda"), 0.3 * r())}


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 3, 31, 64, 257, 511, 1000, 4097, 8192, 20011, 50257])
def test_filters(kind, vocab):
    rows = 24 if vocab < 5000 else 10
    gen = torch.Generator("cuda").manual_seed(vocab)
    logits = (torch.randn(rows, vocab, device="cuda", generator=gen) * 3).to(TYPES[kind])
    uniform = torch.rand(rows, device="cuda", generator=gen)
    check(logits, uniform)
    for name, value in (("temperature", 0.7), ("top_k", 5), ("top_k", max(1, vocab // 2)), ("top_p", 0.9), ("top_p", 0.3), ("min_p", 0.05)):
        check(logits, uniform, **{name: column(rows, value, name)})
    check(logits, uniform, **mixed(rows, gen, vocab))
    check(logits, uniform, **mixed(rows, gen, vocab))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab,pad", [(100, 1), (1000, 3), (33000, 7), (131072, 0), (200003, 0), (300000, 5)])
def test_long_rows_and_strides(kind, vocab, pad):
    rows = 5
    gen = torch.Generator("cuda").manual_seed(vocab)
    logits = torch.full((rows, vocab + pad), float("nan"), device="cuda", dtype=TYPES[kind])
    logits[:, :vocab] = torch.randn(rows, vocab, device="cuda", generator=gen) * 2.5
    logits = logits[:, :vocab]
    uniform = torch.rand(rows, device="cuda", generator=gen)
    check(logits, uniform)
    check(logits, uniform, **mixed(rows, gen, vocab))
    check(logits, uniform, top_p=column(rows, 0.95, "top_p"))
    check(logits, uniform, top_k=column(rows, 50, "top_k"), top_p=column(rows, 0.9, "top_p"), min_p=column(rows, 0.02, "min_p"))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab", [(256, 513), (257, 513), (257, 1000), (300, 2047), (301, 2048), (257, 2049)])
def test_rows_of_medium_length(kind, rows, vocab):
    """Many rows are a wavefront's each, few a workgroup's; with the same tokens."""
    gen = torch.Generator("cuda").manual_seed(vocab)
    logits = (torch.randn(rows, vocab, device="cuda", generator=gen) * 3).to(TYPES[kind])
    logits[7, 3:] = float("-inf")
    uniform = torch.rand(rows, device="cuda", generator=gen)
    settings = mixed(rows, gen, vocab)
    tokens = check(logits, uniform, **settings)
    few, _ = draw(logits[:24], uniform[:24], **{k: v[:24] for k, v in settings.items()})
    assert torch.equal(tokens[:24], few)
    check(logits, uniform, top_k=column(rows, vocab - 1, "top_k"), top_p=column(rows, 0.8, "top_p"))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [5, 300, 9000, 40000])
def test_equal_values(kind, vocab):
    """Ties go to the lower place, in every filter: rows of one value, of two, of a few."""
    gen = torch.Generator("cuda").manual_seed(vocab)
    values = torch.randint(0, 3, (6, vocab), device="cuda", generator=gen).float() * 0.5 - 0.5
    values[0] = 1.25
    values[1] = -3.0
    values[2] = (torch.arange(vocab, device="cuda") % 2).float()
    values[3, ::2] = -0.0
    values[3, 1::2] = 0.0
    logits = values.to(TYPES[kind])
    for u in (0.0, 0.25, 0.5, 1 - 2.0 ** -24):
        uniform = torch.full((6,), u, device="cuda")
        check(logits, uniform)
        for k in (1, 2, vocab // 2, vocab - 1, vocab, vocab + 1):
            check(logits, uniform, top_k=column(6, k, "top_k"))
            check(logits, uniform, top_k=column(6, k, "top_k"), top_p=column(6, 0.5, "top_p"))
        for p in (0.0, -1.0, 1e-9, 0.25, 0.5, 0.75, 1.0, 2.0):
            check(logits, uniform, top_p=column(6, p, "top_p"))
        for m in (-1.0, 0.0, 0.5, 1.0, 7.0):
            check(logits, uniform, min_p=column(6, m, "min_p"))
        assert check(logits, uniform, temperature=column(6, 0.0, "temperature")).tolist() == logits.float().cpu().numpy().argmax(1).tolist()


@pytest.mark.parametrize("kind", TYPES)
def test_masked_entries_and_rows_without_a_distribution(kind):
    dtype, vocab = TYPES[kind], 700
    lowest = torch.finfo(dtype).min
    gen = torch.Generator("cuda").manual_seed(2)
    logits = (torch.randn(16, vocab, device="cuda", generator=gen) * 2).to(dtype)
    logits[0] = -math.inf                               # nothing is left
    logits[1, 3:] = -math.inf
    logits[2] = -math.inf
    logits[2, 77] = -5.0                                # one is
    logits[3] = lowest                                  # a mask of the type's lowest value in every place: all alike
    logits[4, :-1] = lowest
    logits[5, 9] = math.nan
    logits[6, 9] = math.inf
    logits[7] = math.inf
    logits[8, ::2] = -math.inf
    logits[9, 600:] = lowest
    logits[10] = torch.finfo(dtype).max
    logits[11, 0] = torch.finfo(dtype).max
    for u in (0.0, 0.4, 1 - 2.0 ** -24):
        uniform = torch.full((16,), u, device="cuda")
        for s in ({}, dict(top_k=column(16, 10, "top_k")), dict(top_p=column(16, 0.8, "top_p")), dict(min_p=column(16, 0.1, "min_p")),
                  dict(temperature=column(16, 0.0, "temperature")), dict(temperature=column(16, 1e-30, "temperature")),
                  dict(temperature=column(16, 1e30, "temperature")), mixed(16, gen, vocab)):
            tokens = check(logits, uniform, **s)
            assert tokens[[0, 5, 6, 7]].tolist() == [-1] * 4 and tokens[2] == 77 and tokens[4] == vocab - 1
    # such a token masks its row in the calls behind it
    logp = torch.full((16,), 5.0, device="cuda")
    ef.ef_token_logp(logits, tokens, logp)
    assert logp[[0, 5, 6, 7]].tolist() == [0.0] * 4


@pytest.mark.parametrize("kind", TYPES)
def test_many_improbable_entries(kind):
    """Three million entries of e^-22 each, 0.0008 in all beside the one likely one: they are drawn where u says so."""
    vocab = 3000000
    logits = torch.full((4, vocab), -22.0, device="cuda", dtype=TYPES[kind])
    logits[:, 5] = 0.0
    uniform = torch.tensor([0.5, 1 - 2.0 ** -24, 0.9995, 1 - 2.0 ** -12], device="cuda")
    tokens = check(logits, uniform)
    assert tokens[0] == 5 and int(tokens[1]) > vocab - 1000 and 5 < int(tokens[2]) < vocab
    check(logits, uniform, top_p=column(4, 0.9995, "top_p"))
    check(logits, uniform, temperature=column(4, 0.9, "temperature"))


def test_more_rows_than_a_launch_takes():
    """2^22 workgroups to a launch; rows of one entry or two."""
    rows = 4 * (1 << 22) + 9
    logits = torch.zeros(rows, 2, device="cuda", dtype=torch.bfloat16)
    logits[:, 1] = -math.inf
    logits[-3:] = torch.tensor([-math.inf, 0.0], device="cuda")
    tokens, logp = draw(logits, torch.full((rows,), 0.5, device="cuda"))
    assert not tokens[:-3].any() and tokens[-3:].tolist() == [1, 1, 1] and not logp.any()


def test_settings_out_of_range():
    logits = torch.randn(8, 100, device="cuda")
    uniform = torch.full((8,), 0.5, device="cuda")
    nan = math.nan
    bad = torch.tensor([1.0, -0.1, nan, math.inf, 0.5, -0.0, 1 - 2.0 ** -24, 2.0], device="cuda")
    assert (check(logits, bad) < 0).tolist() == [True, True, True, True, False, False, False, True]
    heat = torch.tensor([1.0, -0.1, nan, math.inf, 0.5, -0.0, 1e-45, 3e38], device="cuda")
    assert (check(logits, uniform, temperature=heat) < 0).tolist() == [False, True, True, True, False, False, False, False]
    p = torch.tensor([1.0, -0.1, nan, math.inf, 0.5, -0.0, 1e-45, -math.inf], device="cuda")
    assert (check(logits, uniform, top_p=p) < 0).tolist() == [False, False, True] + [False] * 5
    assert (check(logits, uniform, min_p=p) < 0).tolist() == [False, False, True] + [False] * 5
    k = torch.tensor([0, -1, -2 ** 31, 2 ** 31 - 1, 1, 99, 100, 101], device="cuda", dtype=torch.int32)
    check(logits, uniform, top_k=k)


@pytest.mark.parametrize("kind", TYPES)
def test_logp_is_the_policys(kind):
    """As ef_token_logp has it, whatever the settings: what the policy loss takes for logp_old."""
    gen = torch.Generator("cuda").manual_seed(6)
    logits = (torch.randn(300, 259, device="cuda", generator=gen) * 2).to(TYPES[kind])
    tokens, logp = draw(logits, torch.rand(300, device="cuda", generator=gen), **mixed(300, gen, 259))
    other = torch.empty(300, device="cuda")
    ef.ef_token_logp(logits, tokens, other)
    # that sum is in fp32: some additions and exponentials, and the logarithm's rounding
    assert float((logp - other).abs().max()) <= 130 * 2.0 ** -24 + 4 * 2.0 ** -24 * 20


def test_frequencies():
    """40000 draws from one distribution with its filters: each entry's number within 5 standard deviations of its share."""
    gen = torch.Generator("cuda").manual_seed(9)
    row = torch.randn(40, device="cuda", generator=gen) * 1.5
    n = 40000
    logits = row.expand(n, 40).contiguous()
    tokens, _ = draw(logits, torch.rand(n, device="cuda", generator=gen), temperature=column(n, 0.8, "temperature"), top_k=column(n, 20, "top_k"),
                     top_p=column(n, 0.9, "top_p"))
    v = row.double().cpu().numpy()
    order = np.argsort(-v, kind="stable")[:20]
    w = np.exp((v[order] - v.max()) / 0.8)
    before = np.cumsum(w) - w
    w = np.where(before < 0.9 * w.sum(), w, 0)
    share = np.zeros(40)
    share[order] = w / w.sum()
    seen = torch.bincount(tokens, minlength=40).cpu().numpy()
    assert (np.abs(seen - n * share) <= 5 * np.sqrt(n * share * (1 - share)) + (share > 0)).all()


def test_captured_and_replayed():
    rows, vocab = 20, 5000
    gen = torch.Generator("cuda").manual_seed(4)
    ws, logits, uniform = ef.ef_workspace_create(rows), torch.randn(rows, vocab, device="cuda", generator=gen), torch.rand(rows, device="cuda", generator=gen)
    settings = mixed(rows, gen, vocab)
    tokens, logp = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros(rows, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def step():
        ef.ef_sample_tokens(ws, logits, uniform, *settings.values(), tokens, logp)

    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    for _ in range(3):
        logits.normal_(generator=gen)
        uniform.uniform_(generator=gen)
        step()
        want = tokens.clone(), logp.clone()
        tokens.zero_(), logp.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(logp, want[1])


def test_no_rows():
    ws = ef.ef_workspace_create(0)
    empty = torch.zeros(0, 9, device="cuda")
    ef.ef_sample_tokens(ws, empty, torch.zeros(0, device="cuda"), None, None, None, None, torch.zeros(0, dtype=torch.int64, device="cuda"), None)
