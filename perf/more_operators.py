"""Measured cases of what else a worker's training step is made of: the gated feed-forward block, forward and backward, the
drawing of tokens from logits, and the gradients' norm with clipping into the flat rows that the worker step reads.

A case is a dict of plain values:

  path      which call one pass makes
              gated       ef_gated_forward: both projections, the activation and the product
              gated_back  ef_gated_backward: gradients of the two projections' outputs and of the block's input
              sample      ef_sample_tokens: temperature, top-k, top-p and min-p, tokens from given random numbers
              clip        ef_grad_clip: norm over many tensors, clipped copies in a flat fp32 row for each worker
  type      "bf16" or "fp32": of activations and weights, or of logits; of gradient tensors also "mixed": both in turn
  rows      tokens (gated, gated_back), sequences (sample)
  width     channels of the block's input; entries of the vocabulary (sample)
  inner     channels of the product (gated, gated_back)
  gate      "silu" or "gelu"
  keep      the projections' outputs are kept for the backward pass (gated)
  filters   "none", "top_k", "top_p", "all", or "mixed": every row its own, greedy ones among them (sample)
  padded    entries at the vocabulary's end that are never drawn: their logits are -inf (sample)
  workers   each has a row of its own and clips by itself (clip)
  tensors   a worker's gradient tensors, of very different sizes (clip)
  total     their elements in all
"""
import math
import random

import numpy as np
import torch

own = False     # False: plain torch operations in 32 and 64 bits; True: the library's calls

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
GELU = 2.0 * math.sqrt(2.0 / math.pi)
CUBIC = 0.044715
MAX_NORM = 1.0


# --------------------------------------------------------------------------------------------- cases ---

def listed():
    return [
        # one token of a 1024 wide model being sampled from: every weight read once
        {"name": "gated_token", "path": "gated", "type": "bf16", "rows": 1, "width": 1024, "inner": 4096, "gate": "silu", "keep": False},
        # a training batch: eight sequences of 1024 tokens
        {"name": "gated_batch", "path": "gated", "type": "bf16", "rows": 8192, "width": 1024, "inner": 4096, "gate": "silu", "keep": True},
        # a wider model's prompts, nothing kept
        {"name": "gated_wide", "path": "gated", "type": "bf16", "rows": 8192, "width": 2048, "inner": 8192, "gate": "gelu", "keep": False},
        # the training batch in its backward pass
        {"name": "gated_back_batch", "path": "gated_back", "type": "bf16", "rows": 8192, "width": 1024, "inner": 4096, "gate": "silu"},
        # fp32 at odd sizes: rows that start at any multiple of four bytes
        {"name": "gated_back_odd", "path": "gated_back", "type": "fp32", "rows": 777, "width": 515, "inner": 1031, "gate": "gelu"},
        # one sequence being continued
        {"name": "sample_one", "path": "sample", "type": "bf16", "rows": 1, "width": 50257, "filters": "all", "padded": 0},
        # many sequences at once, each with settings of its own
        {"name": "sample_batch", "path": "sample", "type": "bf16", "rows": 256, "width": 50304, "filters": "mixed", "padded": 47},
        # a large vocabulary in fp32, the nucleus alone
        {"name": "sample_wide", "path": "sample", "type": "fp32", "rows": 64, "width": 128256, "filters": "top_p", "padded": 0},
        # a small vocabulary (bytes and a few more), a policy's own distribution: the rollouts of a training step
        {"name": "sample_bytes", "path": "sample", "type": "fp32", "rows": 4096, "width": 259, "filters": "none", "padded": 0},
        # a small network's gradients of two workers
        {"name": "clip_small", "path": "clip", "type": "fp32", "workers": 2, "tensors": 65, "total": 272474},
        # seven workers of a middle sized one, tensors of either type
        {"name": "clip_workers", "path": "clip", "type": "mixed", "workers": 7, "tensors": 161, "total": 25557032},
        # one worker of a 354 M transformer whose backward pass leaves bf16
        {"name": "clip_transformer", "path": "clip", "type": "bf16", "workers": 1, "tensors": 289, "total": 353772544},
    ]


def spread(rng, low, high):
    """A whole number between the two, spread over their logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    path = rng.choice(("gated", "gated", "gated_back", "gated_back", "sample", "sample", "sample", "clip", "clip"))
    case = {"path": path, "type": rng.choice(("bf16", "fp32"))}
    if path in ("gated", "gated_back"):
        # fp32 products take ten times as long
        most = 8192 if case["type"] == "bf16" else 2048
        case.update(rows=spread(rng, 1, most), width=spread(rng, 24, 2048), inner=spread(rng, 24, most), gate=rng.choice(("silu", "gelu")))
        if path == "gated":
            case["keep"] = rng.random() < 0.5
    elif path == "sample":
        case.update(rows=spread(rng, 1, 256), width=spread(rng, 31, 128256), filters=rng.choice(("none", "top_k", "top_p", "all", "mixed")),
                    padded=0)
        if case["width"] > 1000 and rng.random() < 0.5:
            case["padded"] = rng.randrange(1, 200)
    else:
        case["type"] = rng.choice(("bf16", "fp32", "mixed"))
        tensors = spread(rng, 1, 400)
        case.update(workers=rng.choice((1, 1, 2, 3, 5)), tensors=tensors, total=spread(rng, max(5000, 2 * tensors), 40000000))
    return case


def sizes(case):
    """Elements of a worker's tensors: very different ones, odd ones among them."""
    rng = random.Random(case["tensors"])
    share = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(case["tensors"])]
    each = [1 + int((case["total"] - case["tensors"]) * s / sum(share)) for s in share]
    each[share.index(max(share))] += case["total"] - sum(each)
    return each


def types(case):
    """Their types."""
    if case["type"] == "mixed":
        return [TYPES["fp32" if i % 3 == 1 else "bf16"] for i in range(case["tensors"])]
    return [TYPES[case["type"]]] * case["tensors"]


def work(case):
    path = case["path"]
    if path == "clip":
        read = sum(n * (2 if t is torch.bfloat16 else 4) for n, t in zip(sizes(case), types(case)))
        return {"bytes": case["workers"] * (read + 4 * case["total"] + 4), "flops": 3 * case["workers"] * case["total"]}
    size = 2 if case["type"] == "bf16" else 4
    rows, n = case["rows"], case["width"]
    if path == "sample":
        return {"bytes": rows * (n * size + 32), "flops": 6 * rows * n}
    f = case["inner"]
    if path == "gated":
        moved = rows * n + 2 * f * n + rows * f * (3 if case["keep"] else 1)
    else:
        moved = rows * f * 5 + 2 * f * n + rows * n
    return {"bytes": moved * size, "flops": 4 * rows * n * f}


# ----------------------------------------------------------------------------------- inputs of a pass ---

def settings(case, gen):
    """Temperature, top-k, top-p and min-p of every row; None: not used."""
    rows, kind = case["rows"], case["filters"]

    def rand(low, high):
        return low + (high - low) * torch.rand(rows, device="cuda", generator=gen)

    def some(share, yes, no):
        return torch.where(torch.rand(rows, device="cuda", generator=gen) < share, yes, no)

    one, zero = torch.ones(rows, device="cuda"), torch.zeros(rows, device="cuda")
    if kind == "none":
        return None, None, None, None
    if kind == "top_k":
        return rand(0.6, 1.2), torch.full((rows,), 50, device="cuda", dtype=torch.int32), None, None
    if kind == "top_p":
        return None, None, rand(0.8, 0.95), None
    if kind == "all":
        return rand(0.6, 1.2), torch.full((rows,), 50, device="cuda", dtype=torch.int32), rand(0.8, 0.95), rand(0.01, 0.1)
    k = torch.exp(rand(0.0, math.log(2000.0))).to(torch.int32)
    return (some(0.2, zero, rand(0.5, 1.5)), some(0.5, k, torch.zeros_like(k)), some(0.5, rand(0.5, 0.99), one), some(0.5, rand(0.005, 0.2), zero))


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    path = case["path"]
    s = {"case": case}

    def normal(*shape, sigma=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * sigma

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    if path in ("gated", "gated_back"):
        dtype, rows, n, f = TYPES[case["type"]], case["rows"], case["width"], case["inner"]
        s["w"] = normal(2 * f, n, sigma=n ** -0.5).to(dtype)
        s["pre"] = None
        if path == "gated":
            s["x"] = normal(rows, n).to(dtype)          # the norm's output
            s["z"] = empty(rows, f, dtype=dtype)
            if case["keep"]:
                s["pre"] = empty(rows, 2 * f, dtype=dtype)
        else:
            s["pre"] = normal(rows, 2 * f, sigma=1.2).to(dtype)
            s["dz"] = normal(rows, f, sigma=1e-2).to(dtype)
            s["dz"][torch.rand(rows, device="cuda", generator=gen) < 0.1] = 0       # tokens that the loss masks
            s["dpre"], s["dx"] = empty(rows, 2 * f, dtype=dtype), empty(rows, n, dtype=dtype)
    elif path == "sample":
        rows, n = case["rows"], case["width"]
        live = n - case["padded"]
        logits = normal(rows, n, sigma=2.5)
        likely = torch.randint(0, live, (rows, 24), device="cuda", generator=gen)
        logits.scatter_add_(1, likely, 5.0 + normal(rows, 24, sigma=2.0))          # a few likely ones, sharper or flatter
        logits[:, live:] = -math.inf
        s["logits"] = logits.to(TYPES[case["type"]])
        s["settings"] = settings(case, gen)
        s["uniform"] = torch.rand(rows, device="cuda", generator=gen)
        s["tokens"], s["logp"] = empty(rows, dtype=torch.int64), empty(rows)
    else:
        s["grads"] = []
        for _ in range(case["workers"]):
            # norms on both sides of the limit, a few tensors with much larger entries
            level = MAX_NORM * math.exp(float(torch.rand(1, generator=gen, device="cuda")) * 3.0 - 1.0) / math.sqrt(case["total"])
            s["grads"].append([normal(n, sigma=level * (3.0 if i % 7 == 3 else 1.0)).to(t) for i, (n, t) in enumerate(zip(sizes(case), types(case)))])
        stride = (case["total"] + 3) // 4 * 4
        s["flat"], s["norm"] = torch.zeros(case["workers"], stride, device="cuda"), empty(case["workers"])
    if own:
        import paper_1905_10936_amd as ef
        s["ef"] = ef
        if path != "gated":
            s["workspace"] = ef.ef_workspace_create(case.get("rows", 0))
        if "gate" in case:
            s["gate"] = ef.EF_GATE_SILU if case["gate"] == "silu" else ef.EF_GATE_GELU
    return s


# ------------------------------------------------------------------------------------------- one pass ---

def run(s):
    return (run_own if own else run_plain)(s, s["case"])


def run_own(s, case):
    ef, path = s["ef"], case["path"]
    if path == "gated":
        ef.ef_gated_forward(s["x"], s["w"], s["gate"], s["pre"], s["z"], None)
        return [s["z"], s["pre"]]
    if path == "gated_back":
        ef.ef_gated_backward(s["workspace"], s["dz"], s["pre"], s["w"], s["gate"], s["dpre"], s["dx"])
        return [s["dpre"], s["dx"]]
    if path == "sample":
        ef.ef_sample_tokens(s["workspace"], s["logits"], s["uniform"], *s["settings"], s["tokens"], s["logp"])
        return [s["tokens"], s["logp"]]
    ef.ef_grad_clip(s["workspace"], s["grads"], MAX_NORM, s["flat"], s["norm"])
    return [s["flat"], s["norm"]]


def gate_parts(a, gate):
    """(activation, its derivative)."""
    inner, slope = (a, 1.0) if gate == "silu" else (GELU * (a + CUBIC * a * a * a), GELU * (1.0 + 3.0 * CUBIC * a * a))
    sigma = 1.0 / (1.0 + torch.exp(-inner))
    return a * sigma, sigma + a * sigma * (1.0 - sigma) * slope


def run_plain(s, case):
    path = case["path"]
    if path == "gated":
        both = s["x"].float() @ s["w"].float().t()
        f = case["inner"]
        z = gate_parts(both[:, :f], case["gate"])[0] * both[:, f:]
        return [z.to(s["x"].dtype), both.to(s["x"].dtype) if case["keep"] else None]
    if path == "gated_back":
        f, dtype = case["inner"], s["dz"].dtype
        a, u, dz = s["pre"][:, :f].float(), s["pre"][:, f:].float(), s["dz"].float()
        value, slope = gate_parts(a, case["gate"])
        dpre = torch.cat([dz * u * slope, dz * value], 1).to(dtype)
        return [dpre, (dpre.float() @ s["w"].float()).to(dtype)]
    if path == "sample":
        return sample_plain(s["logits"], s["uniform"], *s["settings"])
    flat, norms = torch.zeros_like(s["flat"]), torch.empty_like(s["norm"])
    for i, grads in enumerate(s["grads"]):
        norm = torch.sqrt(torch.stack([g.double().square().sum() for g in grads]).sum())
        factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)).float()
        at = 0
        for g in grads:
            flat[i, at:at + g.numel()] = g.float() * factor
            at += g.numel()
        norms[i] = norm
    return [flat, norms]


def sample_plain(logits, uniform, temperature, top_k, top_p, min_p):
    """In 64 bits: what is next to a border has to fall on its right side."""
    v = logits.double()
    rows, n = v.shape

    def column(t, other):
        return torch.full((rows, 1), float(other), device=v.device, dtype=torch.float64) if t is None else t.double()[:, None]

    heat, k, p, m = column(temperature, 1.0), column(top_k, 0.0), column(top_p, 1.0), column(min_p, 0.0)
    k = torch.where(heat == 0, torch.ones_like(k), torch.where(k <= 0, torch.full_like(k, float(n)), k))
    heat = torch.where(heat == 0, torch.ones_like(heat), heat)
    gap = v - v.amax(1, keepdim=True)
    w = torch.exp(gap / heat)
    order = torch.sort(v, dim=1, descending=True, stable=True).indices
    sorted_w = w.gather(1, order)
    rank = torch.arange(n, device=v.device)[None, :]
    mass = torch.where(rank < k, sorted_w, torch.zeros_like(sorted_w))
    upto = torch.cumsum(mass, 1)
    keep = (rank < k) & (upto - mass < p * upto[:, -1:]) & (sorted_w >= m)
    keep[:, 0] = True
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, sorted_w, torch.zeros_like(sorted_w)))
    upto = torch.cumsum(kept, 1)
    tokens = (upto <= uniform.double()[:, None] * upto[:, -1:]).sum(1)
    logp = gap.gather(1, tokens[:, None])[:, 0] - torch.log(torch.exp(gap).sum(1))
    return [tokens, logp.float()]


# ------------------------------------------------------------------------------------ in 64 bits, apart ---

def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path == "clip":
        flat = torch.zeros(s["flat"].shape, dtype=torch.float64, device="cuda")
        norms = []
        for row, grads in zip(flat, s["grads"]):
            row[:case["total"]] = torch.cat([g.double() for g in grads])
            norms.append(torch.linalg.vector_norm(row))
            if norms[-1] > MAX_NORM:
                row *= MAX_NORM / norms[-1]
        return [flat, torch.stack(norms)]
    if path == "sample":
        return sample_exact(case, s)
    gate = case["gate"]

    def through(a):
        return a * torch.sigmoid(a) if gate == "silu" else 0.5 * a * (1.0 + torch.tanh(GELU / 2.0 * (a + CUBIC * a.pow(3))))

    w = s["w"].double()
    wg, wu = w[:case["inner"]], w[case["inner"]:]
    if path == "gated":
        x = s["x"].double()
        a, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        return [through(a) * u, torch.cat([a, u], dim=1) if case["keep"] else None]
    a, u = s["pre"].double().chunk(2, dim=1)
    a = a.detach().requires_grad_(True)
    value = through(a)
    slope, = torch.autograd.grad(value.sum(), a)
    da, du = s["dz"].double() * u * slope, s["dz"].double() * value.detach()
    # the input's gradient is that of the projections' as they are stored
    stored = [t.to(s["dz"].dtype).double() for t in (da, du)]
    return [torch.cat([da, du], dim=1), torch.mm(stored[0], wg) + torch.mm(stored[1], wu)]


def sample_exact(case, s):
    v = s["logits"].double().cpu().numpy()
    u = s["uniform"].double().cpu().numpy()
    heat, k, p, m = (None if t is None else t.double().cpu().numpy() for t in s["settings"])
    tokens, logp = [], []
    for i, row in enumerate(v):
        ranked = np.lexsort((np.arange(row.size), -row))
        t = 1.0 if heat is None else heat[i]
        if t == 0.0:
            chosen = int(ranked[0])
        else:
            first = ranked if k is None or k[i] < 1 else ranked[:int(k[i])]
            mass = np.exp((row[first] - row[ranked[0]]) / t)
            before = np.concatenate([[0.0], np.cumsum(mass)])
            stay = len(first) if p is None else int(np.searchsorted(before[:-1], p[i] * before[-1], side="left"))
            if m is not None:
                stay = min(stay, int((mass >= m[i]).sum()))
            stay = np.sort(first[:max(1, stay)])
            mass = np.cumsum(np.exp((row[stay] - row[ranked[0]]) / t))
            chosen = int(stay[np.searchsorted(mass, u[i] * mass[-1], side="right")])
        tokens.append(chosen)
        gap = row - row[ranked[0]]
        logp.append(gap[chosen] - math.log(np.exp(gap).sum()))
    return [torch.tensor(tokens, device="cuda"), torch.tensor(np.array(logp), device="cuda")]
