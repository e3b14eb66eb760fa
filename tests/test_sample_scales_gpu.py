"""Drawing tokens where the filters' bins are far from ordinary: temperatures next to 0 beside logits of any size.  Tokens are filled beforehand (draw), so that one that
was never written shows."""
import pytest
import torch

from tests import train_oracle as oracle
from tests.test_sample_gpu import TYPES, check, column, draw

pytestmark = pytest.mark.gpu

# fp32's 2^100 times the first is beyond its range either way; the others are next to where that begins, and next to the ends of the type
TOPS = (-1e9, 1e9, -2.0 ** 28, 2.0 ** 27, -2.0 ** 20, 2.0 ** 20 - 8192, -1e37, 2e37, -3e38, 3e38, 1e-20, -1e-38, 0.0)


# rows of a wavefront, in LDS, from the caches
@pytest.mark.parametrize("vocab", [300, 9000, 140000])
@pytest.mark.parametrize("kind", TYPES)
def test_temperatures_next_to_0(kind, vocab):
    gen = torch.Generator("cuda").manual_seed(vocab)
    rows = 2 * len(TOPS)
    logits = torch.tensor(TOPS, device="cuda").repeat_interleave(2)[:, None].expand(rows, vocab).contiguous().to(TYPES[kind])
    # every second row: a few values of about that size, and a mask
    for i in range(1, rows, 2):
        t = float(logits[i, 0])
        low = torch.tensor(t * (1.03 if t < 0 else 0.97) - 1.0, device="cuda").to(TYPES[kind])
        logits[i, torch.rand(vocab, device="cuda", generator=gen) < 0.7] = low
        logits[i, :vocab // 3] = float("-inf") if i % 4 == 1 else torch.finfo(TYPES[kind]).min
        logits[i, -2] = t
    for heat in (1e-45, 1e-38, 1e-33, 3.9e-32, 4.3e-32, 1e-30, 1e-9):
        for u in (0.0, 0.6, 1 - 2.0 ** -24):
            uniform = torch.full((rows,), u, device="cuda")
            check(logits, uniform, temperature=column(rows, heat, "temperature"), top_p=column(rows, 0.5, "top_p"))
        check(logits, uniform, temperature=column(rows, heat, "temperature"), top_k=column(rows, vocab // 2, "top_k"), top_p=column(rows, 0.3, "top_p"))
    check(logits, uniform, temperature=column(rows, 3e36, "temperature"), top_p=column(rows, 0.5, "top_p"))


@pytest.mark.parametrize("vocab", [1500, 20000, 140000])
@pytest.mark.parametrize("kind", TYPES)
def test_differences_beyond_fp32(kind, vocab):
    """Logits from one end of the type to the other at a temperature that leaves each its weight: sums are exact, so that the same rows in another place, with the
    log-probabilities or without, have the same tokens, the oracle's.  (The log-probabilities themselves are beyond fp32.)"""
    gen = torch.Generator("cuda").manual_seed(vocab)
    rows, most = 16, torch.finfo(TYPES[kind]).max
    logits = ((torch.rand(rows, vocab, device="cuda", generator=gen, dtype=torch.float64) * 2 - 1) * most).to(TYPES[kind])
    logits[::2] = torch.where(torch.rand(rows // 2, vocab, device="cuda", generator=gen) < 0.5, -most, -0.9 * most).to(TYPES[kind])
    logits[:, 3] = most
    uniform = torch.rand(rows, device="cuda", generator=gen)
    for heat in (3e38, 1e38):
        for p in (1.0, 0.7, 0.2):
            settings = {"temperature": column(rows, heat, "temperature"), "top_p": column(rows, p, "top_p")}
            tokens, logp = draw(logits, uniform, **settings)
            v, u = logits.double().cpu().numpy(), uniform.double().cpu().numpy()
            for i in range(rows):
                assert int(tokens[i]) in oracle.sample(v[i], u[i], heat=float(settings["temperature"][i]), p=float(settings["top_p"][i]))[0], (heat, p, i)
            assert not torch.isnan(logp).any()
            for _ in range(3):
                turned = torch.randperm(rows, device="cuda", generator=gen)
                again, _ = draw(logits[turned], uniform[turned], logp=False, **settings)
                assert torch.equal(again, tokens[turned])
