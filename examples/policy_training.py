"""A small language policy trained by dist-EF-blockSGDM, M workers on one GPU: embedding, a gated feed-forward block if asked for, RMS norm, linear head,
clipped policy loss.

Every worker's forward and backward pass runs on the library's operators, and its gradients land in its row of the flat gradient
that ef_worker_step reads:

    with a block (--inner):
    ef_norm_forward   x = embedding[token] -> y, and xhat in 8 bits: all that the backward pass keeps of the layer's input
    ef_gated_forward  both projections of y -> z, z in 8 bits, and what its backward pass needs
    z @ down^T        (torch) -> added to x by the next norm

    ef_norm_forward   -> y and xhat in 8 bits
    y @ head^T        (torch) -> logits
    ef_sample_tokens  draws the tokens, with their log-probabilities; ef_token_logp  of the reference policy
    ef_policy_loss    loss and, over the logits, their gradient
    ef_weight_grad    head's gradient from the checkpoint, columns times the norm's weight
    dlogits @ head    (torch) -> dy
    ef_norm_backward  embedding rows' gradient from the checkpoint, the norm weight's gradient
    (with a block: dh @ down, ef_gated_backward, two more ef_weight_grad and an ef_norm_backward)
    ef_grad_clip      the worker's row, where its norm is above --clip-norm

    ef_worker_step, ef_server_step, ef_apply: one iteration on the sum of it

The task: token t is followed by (5 t + 1) mod vocab.  The policy draws a next token, is rewarded for the right one, and learns from a batch a few
times over, which is what the clipping is for.

    python examples/policy_training.py [--steps 60] [--workers 4] [--inner 0] [--clip-norm inf]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1905_10936_amd as ef  # noqa: E402

EPS, CLIP, KL = 1e-6, 0.2, 0.01


class Policy:
    """Parameters in one flat fp32 vector, one block each, and the buffers of a pass over `rows` tokens."""

    def __init__(self, vocab, width, rows, seed=0, inner=0):
        self.vocab, self.width, self.rows, self.inner = vocab, width, rows, inner
        self.shapes = {"embedding": (vocab, width), "norm": (width,), "head": (vocab, width)}
        if inner:
            self.shapes.update({"block_norm": (width,), "gate_up": (2 * inner, width), "down": (width, inner)})
        self.offsets = np.concatenate([[0], np.cumsum([int(np.prod(shape)) for shape in self.shapes.values()])])
        self.d = int(self.offsets[-1])
        self.params = torch.zeros((self.d + 3) // 4 * 4, device="cuda")[:self.d]
        p = self.views(self.params)
        gen = torch.Generator("cuda").manual_seed(seed)
        p["embedding"].normal_(0.0, 1.0, generator=gen)
        p["norm"].fill_(1.0)
        p["head"].normal_(0.0, width ** -0.5, generator=gen)
        if inner:
            p["block_norm"].fill_(1.0)
            p["gate_up"].normal_(0.0, width ** -0.5, generator=gen)
            p["down"].normal_(0.0, inner ** -0.5, generator=gen)
        self.workspace = ef.ef_workspace_create(rows)

        def empty(*shape, dtype=torch.float32):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        self.y, self.dx = (empty(rows, width, dtype=torch.bfloat16) for _ in range(2))
        self.act, self.rstd = empty(ef.ef_act_bytes(rows, width), dtype=torch.uint8), empty(rows)
        self.logp, self.losses, self.loss = empty(rows), empty(rows), empty(1)
        if inner:
            self.block_act, self.block_rstd = torch.empty_like(self.act), empty(rows)
            self.pre, self.z = empty(rows, 2 * inner, dtype=torch.bfloat16), empty(rows, inner, dtype=torch.bfloat16)
            self.z_act, self.dh = empty(ef.ef_act_bytes(rows, inner), dtype=torch.uint8), torch.empty_like(self.dx)

    def views(self, flat):
        """The blocks of a flat vector as the matrices they are."""
        return {name: flat[self.offsets[k]:self.offsets[k + 1]].view(shape) for k, (name, shape) in enumerate(self.shapes.items())}

    def logits(self, tokens, params=None):
        """bf16 logits of the next token; leaves the checkpoints and rstd of the norms behind, and what the block keeps."""
        p = self.views(self.params if params is None else params)
        x, residual = p["embedding"][tokens].bfloat16(), None
        if self.inner:
            ef.ef_norm_forward(x, None, p["block_norm"], EPS, None, self.y, self.block_act, self.block_rstd)
            ef.ef_gated_forward(self.y, p["gate_up"].bfloat16(), ef.EF_GATE_SILU, self.pre, self.z, self.z_act)
            x, residual = self.z @ p["down"].bfloat16().t(), x
        ef.ef_norm_forward(x, residual, p["norm"], EPS, None, self.y, self.act, self.rstd)
        return self.y @ p["head"].bfloat16().t()

    def step(self, tokens, actions, old, ref, advantage, weight, grad):
        """Loss of a batch; its gradient goes to `grad`, a row of the workers' flat gradients."""
        p, g = self.views(self.params), self.views(grad)
        logits = self.logits(tokens)
        ef.ef_policy_loss(self.workspace, logits, actions, old, ref, advantage, weight, CLIP, CLIP, KL, self.logp, self.losses, self.loss, logits)
        dlogits = logits                                            # the gradient is written over the logits
        ef.ef_weight_grad(self.workspace, dlogits, self.act, p["norm"], g["head"])
        dy = dlogits @ p["head"].bfloat16()
        ef.ef_norm_backward(self.workspace, dy, self.act, self.rstd, p["norm"], None, self.dx, g["norm"])
        if self.inner:
            dh = self.dh.copy_(self.dx)                             # of the block's output and of the residual alike
            ef.ef_weight_grad(self.workspace, dh, self.z_act, None, g["down"])
            dpre, dy = self.pre, torch.empty_like(dh)               # the gradient is written over what the block kept
            ef.ef_gated_backward(self.workspace, dh @ p["down"].bfloat16(), self.pre, p["gate_up"].bfloat16(), ef.EF_GATE_SILU, dpre, dy)
            ef.ef_weight_grad(self.workspace, dpre, self.block_act, p["block_norm"], g["gate_up"])
            ef.ef_norm_backward(self.workspace, dy, self.block_act, self.block_rstd, p["block_norm"], dh, self.dx, g["block_norm"])
        g["embedding"].zero_().index_add_(0, tokens, self.dx.float())
        return self.loss


def train(steps=60, workers=4, vocab=259, width=96, rows=1024, epochs=2, eta=0.3, mu=0.9, seed=0, say=print, inner=0, clip_norm=math.inf):
    """Returns the mean reward of every step."""
    policy = Policy(vocab, width, rows, seed, inner)
    plan = ef.ef_plan_create(policy.offsets, workers)
    stride = (policy.d + 3) // 4 * 4
    grad, mom, err = (torch.zeros(workers, stride, device="cuda") for _ in range(3))
    server_err = torch.zeros(policy.d, device="cuda")
    signs, scales = torch.zeros(workers, plan.W, dtype=torch.int64, device="cuda"), torch.zeros(workers, plan.B, device="cuda")
    out_signs, out_scales = torch.zeros(plan.W, dtype=torch.int64, device="cuda"), torch.zeros(plan.B, device="cuda")
    reference = policy.params.clone()
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    norms = torch.zeros(workers, device="cuda")
    eta_prev, rewards = 0.0, []
    for step in range(steps):
        batches = []
        for _ in range(workers):
            tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
            old, ref = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            actions, uniform = torch.empty_like(tokens), torch.rand(rows, device="cuda", generator=gen)
            ef.ef_sample_tokens(policy.workspace, policy.logits(tokens), uniform, None, None, None, None, actions, old)
            ef.ef_token_logp(policy.logits(tokens, reference), actions, ref)
            reward = (actions == (5 * tokens + 1) % vocab).float()
            weight = (torch.rand(rows, device="cuda", generator=gen) < 0.9).float()         # a masked tenth
            batches.append((tokens, actions, old, ref, reward, weight / weight.sum()))
        rewards.append(float(torch.stack([b[4].mean() for b in batches]).mean()))
        for _ in range(epochs):
            loss = 0.0
            for i, (tokens, actions, old, ref, reward, weight) in enumerate(batches):
                advantage = (reward - reward.mean()) / (reward.std() + 1e-3)
                loss += float(policy.step(tokens, actions, old, ref, advantage, weight, grad[i][:policy.d])) / workers
            if clip_norm < math.inf:
                ef.ef_grad_clip(policy.workspace, [[row[:policy.d]] for row in grad], clip_norm, None, norms)
            ef.ef_worker_step(plan, grad, mom, err, mu, eta_prev, eta, signs, scales)
            ef.ef_server_step(plan, workers, signs, scales, server_err, eta_prev, eta, out_signs, out_scales)
            ef.ef_apply(plan, policy.params, out_signs, out_scales, eta)
            eta_prev = eta
        if say and (step % 10 == 0 or step == steps - 1):
            say("step %3d  reward %.3f  loss %+.4f" % (step, rewards[-1], loss), flush=True)
    return rewards


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--workers", type=int, default=4)
    parser.add_argument("--inner", type=int, default=0)
    parser.add_argument("--clip-norm", type=float, default=math.inf)
    a = parser.parse_args()
    train(steps=a.steps, workers=a.workers, inner=a.inner, clip_norm=a.clip_norm)
