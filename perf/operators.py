"""Measured cases of the operators a worker's forward and backward pass is made of: RMS norm with an output in 8 bits, 8-bit
activation checkpoints and the weight gradient taken from them, and the clipped policy loss on logits.

A case is a dict of plain values:

  path      which call one pass makes
              norm       ef_norm_forward: residual's addition, norm, 8-bit checkpoint of the normalised rows
              norm_back  ef_norm_backward from the checkpoint: gradients of the rows and of the weight
              encode     ef_act_encode
              decode     ef_act_decode
              grad       ef_weight_grad: the weight gradient of a linear layer from its input's checkpoint
              loss       ef_policy_loss: loss and gradient with respect to the logits
              logp       ef_token_logp
  type      "bf16" or "fp32": of the activations, logits and their gradients (parameters and their gradients are fp32)
  rows      tokens
  width     channels (norm, checkpoint), the linear layer's input (grad), entries of the vocabulary (loss, logp)
  out       the linear layer's output (grad)
  residual  the norm adds one / the backward pass has its gradient
  scaled    the layer's input is the checkpoint times the norm's weight (grad)
  padded    entries at the vocabulary's end that are never drawn: their logits are -inf (loss, logp)
"""
import math

import torch

own = False     # False: plain torch operations in 32 bits; True: the library's calls

EPS = 1e-6
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
GROUP = 32      # channels to a scale


# --------------------------------------------------------------------------------------------- cases ---

def listed():
    return [
        # one token of a 1024 wide model being sampled from: the call's latency
        {"name": "norm_token", "path": "norm", "type": "bf16", "rows": 1, "width": 1024, "residual": True},
        # a training batch of the 354 M transformer: sixteen sequences of 1024 tokens
        {"name": "norm_batch", "path": "norm", "type": "bf16", "rows": 16384, "width": 1024, "residual": True},
        # the same in its backward pass
        {"name": "norm_back_batch", "path": "norm_back", "type": "bf16", "rows": 16384, "width": 1024, "residual": True},
        # fp32 activations, no residual, rows that start at any multiple of four bytes
        {"name": "norm_back_odd", "path": "norm_back", "type": "fp32", "rows": 1537, "width": 1031, "residual": False},
        # checkpoint of the inner layer's activations (ff 4096), and reading it back
        {"name": "encode_inner", "path": "encode", "type": "bf16", "rows": 16384, "width": 4096},
        {"name": "decode_inner", "path": "decode", "type": "bf16", "rows": 16384, "width": 4096},
        # weight gradient of the inner layer
        {"name": "grad_inner", "path": "grad", "type": "bf16", "rows": 8192, "width": 1024, "out": 4096, "scaled": True},
        # and of the head over the vocabulary: the largest product of the step
        {"name": "grad_head", "path": "grad", "type": "bf16", "rows": 8192, "width": 1024, "out": 50257, "scaled": True},
        # fp32 gradients at odd sizes
        {"name": "grad_odd", "path": "grad", "type": "fp32", "rows": 777, "width": 1031, "out": 515, "scaled": False},
        # policy loss over a batch: every logit read once, every gradient written once
        {"name": "loss_batch", "path": "loss", "type": "bf16", "rows": 4096, "width": 50257, "padded": 0},
        # a handful of tokens in fp32, the vocabulary's end padded
        {"name": "loss_few", "path": "loss", "type": "fp32", "rows": 5, "width": 50304, "padded": 47},
        # a small vocabulary (bytes and a few more), long sequences
        {"name": "loss_bytes", "path": "loss", "type": "fp32", "rows": 32768, "width": 259, "padded": 0},
    ]


def spread(rng, low, high):
    """A whole number between the two, spread over their logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    path = rng.choice(("norm", "norm_back", "encode", "decode", "grad", "grad", "loss", "loss", "logp"))
    case = {"path": path, "type": rng.choice(("bf16", "fp32"))}
    if path in ("norm", "norm_back"):
        case.update(rows=spread(rng, 1, 16384), width=spread(rng, 24, 8192), residual=rng.random() < 0.7)
    elif path in ("encode", "decode"):
        case.update(rows=spread(rng, 1, 16384), width=spread(rng, 24, 8192))
    elif path == "grad":
        case.update(rows=spread(rng, 1, 8192), width=spread(rng, 24, 2048), out=spread(rng, 24, 8192), scaled=rng.random() < 0.5)
    else:
        case.update(rows=spread(rng, 1, 4096), width=spread(rng, 31, 60000), padded=0)
        if case["width"] > 1000 and rng.random() < 0.5:
            case["padded"] = rng.randrange(1, 200)
    if case.get("width", 0) % 1024 == 0:    # the listed ones have those
        case["width"] += 1
    return case


def work(case):
    size = 2 if case["type"] == "bf16" else 4
    rows, n = case["rows"], case["width"]
    act = rows * (n + (n + GROUP - 1) // GROUP)
    path = case["path"]
    if path == "norm":
        moved = 4 if case["residual"] else 2       # x, y; the residual and the sum
        return {"bytes": rows * n * size * moved + act + 4 * n + 4 * rows, "flops": 8 * rows * n}
    if path == "norm_back":
        moved = 3 if case["residual"] else 2
        return {"bytes": rows * n * size * moved + act + 8 * n + 4 * rows, "flops": 10 * rows * n}
    if path in ("encode", "decode"):
        return {"bytes": rows * n * size + act, "flops": 2 * rows * n}
    if path == "grad":
        m = case["out"]
        return {"bytes": rows * m * size + act + 4 * m * n + (4 * n if case["scaled"] else 0), "flops": 2 * rows * m * n}
    if path == "loss":
        return {"bytes": 2 * rows * n * size + rows * 32, "flops": 8 * rows * n}
    return {"bytes": rows * n * size + rows * 12, "flops": 4 * rows * n}


# -------------------------------------------------------------------------- the checkpoint's format ---

def act_layout(rows, n):
    """(bytes a row of codes takes, scales a row has, where the scales start, bytes in all)."""
    groups = (n + GROUP - 1) // GROUP
    at = rows * groups * GROUP
    return groups * GROUP, groups, at, (at + rows * groups + 15) // 16 * 16


def scale_bytes(largest):
    """Exponents (biased by 127) of the groups' scales: the least power of two that brings the largest value to 448 or below."""
    f, k = torch.frexp(largest)
    e = k - 9 + (f > 0.875).to(k.dtype)
    return torch.where(largest > 0, e, torch.full_like(e, -117)).clamp(-117, 119) + 127


def power(byte):
    """2^(byte - 127) in 32 bits."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def encoded(v):
    """(codes as e4m3 numbers [rows][padded n], scales as powers of two in 8 bits [rows][groups]) of a matrix in 32 bits."""
    rows, n = v.shape
    padded, groups = act_layout(rows, n)[:2]
    v = torch.nn.functional.pad(v, (0, padded - n)).view(rows, groups, GROUP)
    byte = scale_bytes(v.abs().amax(-1))
    codes = (v * power(254 - byte)[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes.view(rows, padded), byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def parts(act, rows, n):
    """The two parts of a checkpoint's buffer, as what encoded() gives."""
    padded, groups, at, _ = act_layout(rows, n)
    return (act[:at].view(torch.float8_e4m3fn).view(rows, padded),
            act[at:at + rows * groups].view(torch.float8_e8m0fnu).view(rows, groups))


def decoded(act, rows, n):
    """A checkpoint's values in 32 bits."""
    codes, scales = parts(act, rows, n)
    return (codes.float().view(rows, -1, GROUP) * power(scales.view(torch.uint8))[..., None]).view(rows, -1)[:, :n]


# ----------------------------------------------------------------------------------- inputs of a pass ---

def activations(gen, rows, n, dtype):
    """Normal values, a few channels with much larger ones."""
    v = torch.randn(rows, n, device="cuda", generator=gen)
    v[:, :: max(1, n // 5)] *= 12.0
    return v.to(dtype)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dtype, rows, n, path = TYPES[case["type"]], case["rows"], case["width"], case["path"]
    s = {"case": case}

    def normal(*shape, sigma=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * sigma

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    if path in ("norm", "norm_back", "grad"):
        s["weight"] = 1.0 + normal(n, sigma=0.1)
    if path in ("norm", "encode"):
        s["x"] = activations(gen, rows, n, dtype)
        s["act"] = torch.zeros(act_layout(rows, n)[3], device="cuda", dtype=torch.uint8)
    if path == "norm":
        s["residual"] = activations(gen, rows, n, dtype) if case["residual"] else None
        s["h"] = empty(rows, n, dtype=dtype) if case["residual"] else None
        s["y"], s["rstd"] = empty(rows, n, dtype=dtype), empty(rows)
    if path in ("norm_back", "decode", "grad"):
        v = activations(gen, rows, n, torch.float32)
        rstd = 1.0 / torch.sqrt((v * v).mean(-1) + EPS)
        codes, scales = encoded(v * rstd[:, None])
        _, _, at, size = act_layout(rows, n)
        s["act"] = torch.zeros(size, device="cuda", dtype=torch.uint8)
        s["act"][:at] = codes.view(torch.uint8).view(-1)
        s["act"][at:at + scales.numel()] = scales.view(torch.uint8).view(-1)
        s["rstd"] = rstd
        del v, codes, scales
    if path == "norm_back":
        s["dy"] = normal(rows, n, sigma=1e-2).to(dtype)
        s["dh"] = normal(rows, n, sigma=1e-2).to(dtype) if case["residual"] else None
        s["dx"], s["dweight"] = empty(rows, n, dtype=dtype), empty(n)
    if path == "decode":
        s["y"] = empty(rows, n, dtype=dtype)
    if path == "grad":
        s["dz"] = normal(rows, case["out"], sigma=1e-3).to(dtype)
        s["dz"][torch.rand(rows, device="cuda", generator=gen) < 0.1] = 0       # tokens that the loss masks
        s["dw"] = empty(case["out"], n)
    if path in ("loss", "logp"):
        live = n - case["padded"]
        logits = normal(rows, n, sigma=2.0)
        s["tokens"] = torch.randint(0, live, (rows,), device="cuda", generator=gen)
        logits.scatter_add_(1, s["tokens"][:, None], normal(rows, 1, sigma=2.0) + 7.0)     # drawn tokens are likely ones
        logits[:, live:] = -math.inf
        s["logits"] = logits.to(dtype)
        del logits
        s["logp"] = empty(rows)
    if path == "loss":
        chosen = logits_of(s["logits"], s["tokens"])
        s["old"], s["ref"] = chosen + normal(rows, sigma=0.15), chosen + normal(rows, sigma=0.3)
        s["advantage"] = normal(rows)
        keep = (torch.rand(rows, device="cuda", generator=gen) < 0.9).float()
        keep[0] = 1.0
        s["token_weight"] = keep / keep.sum()
        s["losses"], s["loss"], s["dlogits"] = empty(rows), empty(1), empty(rows, n, dtype=dtype)
    if own:
        import paper_1905_10936_amd as ef
        s["ef"] = ef
        if path in ("norm_back", "grad", "loss"):
            s["workspace"] = ef.ef_workspace_create(rows)
    return s


def logits_of(logits, tokens):
    """Log-probabilities of the tokens, in 32 bits."""
    v = logits.float()
    top = v.amax(-1, keepdim=True)
    total = torch.exp(v - top).sum(-1)
    return (v.gather(1, tokens[:, None]) - top)[:, 0] - torch.log(total)


# ------------------------------------------------------------------------------------------- one pass ---

def run(s):
    case = s["case"]
    return (run_own if own else run_plain)(s, case["path"], case["rows"], case["width"], TYPES[case["type"]])


def run_own(s, path, rows, n, dtype):
    ef = s["ef"]
    if path == "norm":
        ef.ef_norm_forward(s["x"], s["residual"], s["weight"], EPS, s["h"], s["y"], s["act"], s["rstd"])
        return [s["h"], s["y"], s["rstd"], *parts(s["act"], rows, n)]
    if path == "norm_back":
        ef.ef_norm_backward(s["workspace"], s["dy"], s["act"], s["rstd"], s["weight"], s["dh"], s["dx"], s["dweight"])
        return [s["dx"], s["dweight"]]
    if path == "encode":
        ef.ef_act_encode(s["x"], s["act"])
        return list(parts(s["act"], rows, n))
    if path == "decode":
        ef.ef_act_decode(s["act"], s["y"])
        return s["y"]
    if path == "grad":
        ef.ef_weight_grad(s["workspace"], s["dz"], s["act"], s["weight"] if s["case"]["scaled"] else None, s["dw"])
        return s["dw"]
    if path == "logp":
        ef.ef_token_logp(s["logits"], s["tokens"], s["logp"])
        return s["logp"]
    ef.ef_policy_loss(s["workspace"], s["logits"], s["tokens"], s["old"], s["ref"], s["advantage"], s["token_weight"], CLIP_LOW,
                      CLIP_HIGH, KL, s["logp"], s["losses"], s["loss"], s["dlogits"])
    return [s["loss"], s["losses"], s["logp"], s["dlogits"]]


def run_plain(s, path, rows, n, dtype):
    if path == "norm":
        v = s["x"].float()
        if s["residual"] is not None:
            v = v + s["residual"].float()
        rstd = 1.0 / torch.sqrt((v * v).mean(-1) + EPS)
        xhat = v * rstd[:, None]
        return [None if s["residual"] is None else v.to(dtype), (xhat * s["weight"]).to(dtype), rstd, *encoded(xhat)]
    if path == "norm_back":
        xhat, dy = decoded(s["act"], rows, n), s["dy"].float()
        g = dy * s["weight"]
        dx = (g - xhat * (g * xhat).mean(-1, keepdim=True)) * s["rstd"][:, None]
        if s["dh"] is not None:
            dx = s["dh"].float() + dx
        return [dx.to(dtype), (dy * xhat).sum(0)]
    if path == "encode":
        return list(encoded(s["x"].float()))
    if path == "decode":
        return decoded(s["act"], rows, n).to(dtype)
    if path == "grad":
        dw = s["dz"].float().t() @ decoded(s["act"], rows, n)
        return dw * s["weight"] if s["case"]["scaled"] else dw
    if path == "logp":
        return logits_of(s["logits"], s["tokens"])
    v, tokens, weight, advantage = s["logits"].float(), s["tokens"], s["token_weight"], s["advantage"]
    live = weight != 0
    e = torch.exp(v - v.amax(-1, keepdim=True))
    total = e.sum(-1)
    logp = torch.where(live, (v.gather(1, tokens[:, None]) - v.amax(-1, keepdim=True))[:, 0] - torch.log(total), torch.zeros_like(total))
    ratio = torch.exp(logp - s["old"])
    free, held = ratio * advantage, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * advantage
    d = s["ref"] - logp
    losses = torch.where(live, weight * (KL * (torch.expm1(d) - d) - torch.minimum(free, held)), torch.zeros_like(total))
    slope = torch.where(live, weight * (-torch.where(free <= held, free, torch.zeros_like(free)) - KL * torch.expm1(d)), torch.zeros_like(total))
    dlogits = e * (-slope / total)[:, None]
    dlogits.scatter_add_(1, tokens[:, None], slope[:, None])
    return [losses.sum().view(1), losses, logp, dlogits.to(dtype)]


# ------------------------------------------------------------------------------------ in 64 bits, apart ---

def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.dtype in (torch.float32, torch.bfloat16)}
    rows, n, path = case["rows"], case["width"], case["path"]

    def quantised(v):
        """e4m3 numbers and powers of two, by their definitions."""
        full, groups = act_layout(rows, n)[:2]
        t = v.new_zeros(rows, full)
        t[:, :n] = v
        t = t.view(rows, groups, GROUP)
        top = t.abs().amax(2)
        e = torch.ceil(torch.log2((top / 448.0).clamp(min=2.0 ** -130)))
        e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)        # what the logarithm's rounding has moved
        e = torch.where(448.0 * torch.exp2(e) < top, e + 1, e).clamp(-117, 119)
        t = (t / torch.exp2(e)[:, :, None]).clamp(-448, 448)
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        return [(torch.round(t / step) * step).view(rows, full), torch.exp2(e)]

    def values():
        codes, scales = parts(s["act"], rows, n)
        e = scales.view(torch.uint8).double() - 127
        return (codes.double() * torch.exp2(e).repeat_interleave(GROUP, dim=1))[:, :n]

    if path == "encode":
        return quantised(d["x"])
    if path == "norm":
        total = d["x"] + d["residual"] if case["residual"] else d["x"]
        rstd = (total.pow(2).sum(1) / n + EPS).pow(-0.5)
        unit = total * rstd.unsqueeze(1)
        return [total if case["residual"] else None, unit * d["weight"], rstd] + quantised(unit)
    if path == "decode":
        return values()
    if path == "grad":
        x = values()
        if case["scaled"]:
            x = x * d["weight"]
        return torch.mm(d["dz"].t(), x)
    if path == "norm_back":
        x = values()
        g = d["dy"] * d["weight"]
        dx = d["rstd"].unsqueeze(1) * (g - x * ((g * x).sum(1, keepdim=True) / n))
        return [dx + d["dh"] if case["residual"] else dx, (d["dy"] * x).sum(0)]
    at = s["tokens"].unsqueeze(1)
    logp = torch.log_softmax(d["logits"], 1)
    chosen = logp.gather(1, at).squeeze(1)
    if path == "logp":
        return chosen
    q, adv = d["token_weight"], d["advantage"]
    masked = q == 0
    ratio = (chosen - d["old"]).exp()
    bound = torch.where(adv >= 0, torch.full_like(adv, 1.0 + CLIP_HIGH), torch.full_like(adv, 1.0 - CLIP_LOW))
    outside = torch.where(adv >= 0, ratio > bound, ratio < bound)
    gap = d["ref"] - chosen
    losses = q * (KL * (torch.expm1(gap) - gap) - adv * torch.where(outside, bound, ratio))
    slope = q * (KL * (1 - gap.exp()) - adv * torch.where(outside, torch.zeros_like(ratio), ratio))
    dlogits = -logp.exp() * slope.unsqueeze(1)
    dlogits.scatter_(1, at, (slope * (1 - chosen.exp())).unsqueeze(1))
    losses, chosen = losses.masked_fill(masked, 0.0), chosen.masked_fill(masked, 0.0)
    return [losses.sum().reshape(1), losses, chosen, dlogits.masked_fill(masked.unsqueeze(1), 0.0)]
