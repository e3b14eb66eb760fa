"""Drawing tokens from rows with one likely entry and very many improbable ones: together they have some steps of a float's uniform, and are drawn where it says so."""
import pytest
import torch

from tests.test_sample_gpu import TYPES, check, column, draw

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24


# (rows, entries, the improbable ones' logit): rows that a wavefront has and that a workgroup has, in LDS and from the caches; next to 1024 and to 131072 entries.  The
# improbable entries have 7.5 to 700 steps.
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab,low", [(300, 500, -20.0), (5, 1024, -21.0), (5, 1025, -21.0), (300, 1500, -21.5), (5, 20011, -23.25), (5, 50257, -24.5), (5, 50257, -25.625),
                                            (5, 128256, -24.5), (5, 131072, -24.5), (5, 131072, -23.25), (5, 131073, -23.25)])
def test_many_improbable_entries(kind, rows, vocab, low):
    values = torch.full((rows, vocab), low, device="cuda")
    values[:, 5] = 0.0
    share = (vocab - 1) * float(torch.tensor(low, dtype=torch.float64).exp())
    steps = int(share / STEP)
    assert steps >= 6
    # from a step into the improbable ones' share to its end, and next before it
    uniform = 1 - STEP * torch.linspace(1, steps - 3, rows, dtype=torch.float64).floor().cuda()
    uniform[-1] = 1 - STEP * (steps + 4)
    uniform = uniform.float()
    logits = values.to(TYPES[kind])
    for settings in ({}, {"top_p": 1 - 2 * STEP}, {"top_k": vocab - 1}, {"min_p": 1e-13}):
        tokens = check(logits, uniform, **{k: column(rows, v, k) for k, v in settings.items()})
        assert bool((tokens[:-1] != 5).all()) and tokens[-1] <= 5, settings
    # another temperature, with the log-probabilities and without them
    heated = (values * 2).to(TYPES[kind])
    assert torch.equal(heated.double(), values.double() * 2)
    for settings in ({"temperature": 2.0}, {"temperature": 2.0, "top_p": 1 - 2 * STEP}):
        settings = {k: column(rows, v, k) for k, v in settings.items()}
        tokens = check(heated, uniform, **settings)
        assert bool((tokens[:-1] != 5).all()) and tokens[-1] <= 5
        assert torch.equal(tokens, draw(heated, uniform, logp=False, **settings)[0])
