"""The example that runs the operators together: its gradients against torch's own, and that it learns."""
import os
import sys

import pytest
import torch

import paper_1905_10936_amd as ef

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_gradients_of_a_worker():
    """E4M3 rounds each value of the checkpoint by up to 2^-4, a fortieth in the mean square, independently: so much of a gradient's norm, and the bf16
    steps 2^-8 each."""
    import policy_training as example
    policy = example.Policy(vocab=131, width=96, rows=500, seed=3)
    gen = torch.Generator("cuda").manual_seed(4)
    tokens, actions = (torch.randint(0, 131, (500,), device="cuda", generator=gen) for _ in range(2))
    old, ref = torch.empty(500, device="cuda"), torch.empty(500, device="cuda")
    ef.ef_token_logp(policy.logits(tokens), actions, old)
    ref.copy_(old - 0.2)
    old += 0.1 * torch.randn(500, device="cuda", generator=gen)
    advantage = torch.randn(500, device="cuda", generator=gen)
    weight = torch.full((500,), 1 / 400.0, device="cuda")
    weight[::5] = 0.0
    grad = torch.full((policy.d,), float("nan"), device="cuda")
    loss = float(policy.step(tokens, actions, old, ref, advantage, weight, grad))

    flat = policy.params.clone().requires_grad_(True)
    p = policy.views(flat)
    x = p["embedding"][tokens]
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + example.EPS) * p["norm"]
    logp = torch.log_softmax(y @ p["head"].t(), 1).gather(1, actions[:, None])[:, 0]
    ratio = torch.exp(logp - old)
    d = ref - logp
    want = -torch.minimum(ratio * advantage, ratio.clamp(1 - example.CLIP, 1 + example.CLIP) * advantage) + example.KL * (torch.expm1(d) - d)
    want = (weight * want).sum()
    want.backward()
    assert abs(loss - float(want.detach())) <= 0.02 * float((weight * advantage.abs()).sum())
    for name, got in policy.views(grad).items():
        exact = policy.views(flat.grad)[name]
        assert float((got - exact).norm()) <= 0.06 * float(exact.norm()), name


def test_it_learns():
    import policy_training as example
    rewards = example.train(steps=25, workers=2, say=None)
    assert rewards[0] < 0.02 and rewards[-1] > 0.1
