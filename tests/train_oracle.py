"""The gated block, the drawing of tokens and clipping by their definitions, in 64 bits on the CPU (NumPy), and the bounds that the library's arithmetic
keeps to.  Shares nothing with the library."""
import math

import numpy as np

EPS = 2.0 ** -24        # half a unit in the last place of fp32
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": EPS}


def inner_slope(a, gate):
    """F(a), F'(a)."""
    if gate == "silu":
        return a, np.ones_like(a)
    c = 2.0 * math.sqrt(2.0 / math.pi)
    return c * (a + 0.044715 * a ** 3), c * (1.0 + 3 * 0.044715 * a * a)


def activation(a, gate):
    """act(a), act'(a), and the relative error that fp32 makes in either: F is rounded in a few places, which moves the exponential by as much of itself as F
    is large; the rest are a handful of roundings."""
    s, ds = inner_slope(a, gate)
    with np.errstate(over="ignore"):
        small = np.exp(-np.abs(s))
    big = 1.0 / (1.0 + small)
    sig = np.where(s < 0, small * big, big)
    return a * sig, sig + a * small * big * big * ds, (np.minimum(np.abs(s), 100.0) + 8) * 4 * EPS


def gated_forward(x, w, gate, kind):
    """z, pre, and how far each may be off.  A sum of n products is n additions, each of which may lose two half units of the sum of sizes so far."""
    f, n = w.shape[0] // 2, w.shape[1]
    pre = x @ w.T
    off = 2 * EPS * n * (np.abs(x) @ np.abs(w).T)
    a, u, a_off, u_off = pre[:, :f], pre[:, f:], off[:, :f], off[:, f:]
    act, _, rel = activation(a, gate)
    # |act'| <= 1.13 for both
    z, z_off = act * u, 1.13 * a_off * (np.abs(u) + u_off) + np.abs(act) * u_off
    z_off = z_off + (np.abs(act * u) + z_off) * rel
    step = HALF_STEP[kind]
    tiny = 2.0 ** -126      # below the least normal number the exponential may be 0
    return z, pre, z_off, z_off + (np.abs(z) + z_off) * step + tiny * (1 + np.abs(u)), off + (np.abs(pre) + off) * step + tiny


def gated_slopes(dz, pre, gate, kind):
    f = dz.shape[1]
    a, u = pre[:, :f], pre[:, f:]
    act, slope, rel = activation(a, gate)
    # act' is a difference where a is negative: its parts' size counts
    s, ds = inner_slope(a, gate)
    with np.errstate(over="ignore"):
        small = np.exp(-np.abs(s))
    big = 1.0 / (1.0 + small)
    size = np.where(s < 0, small * big, big) + np.abs(a) * small * big * big * ds
    out = np.concatenate([dz * u * slope, dz * act], 1)
    off = np.concatenate([np.abs(dz * u) * size * 2 * rel, np.abs(dz * act) * rel], 1)
    return out, off + (np.abs(out) + off) * HALF_STEP[kind] + 2.0 ** -126 * (1 + np.abs(np.concatenate([u, a], 1)))


def input_grad(dpre, w, kind):
    out = dpre @ w
    off = 2 * EPS * w.shape[0] * (np.abs(dpre) @ np.abs(w))
    return out, off + (np.abs(out) + off) * HALF_STEP[kind] + 2.0 ** -126


def sample(v, u, heat=1.0, k=0, p=1.0, m=0.0):
    """(tokens that are right, logp by token): one token, or those within 1e-9 of the whole from u, where it is next to a border."""
    if np.isnan(v).any() or v.max() in (math.inf, -math.inf) or not 0 <= u < 1 or not 0 <= heat < math.inf or math.isnan(p) or math.isnan(m):
        return {-1}, {-1: math.nan}
    order = np.lexsort((np.arange(v.size), -v))
    top = v[order[0]]
    whole = np.exp(v - top).sum()
    logp = lambda t: float(v[t] - top) - math.log(whole)      # noqa: E731
    if heat == 0 or p <= 0:
        return {int(order[0])}, {int(order[0]): logp(order[0])}
    first = order if k <= 0 else order[:int(k)]
    with np.errstate(over="ignore"):
        w = np.exp((v[first] - top) / heat)
    before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
    right = set()
    # the cut of top-p, and neighbours of it that are as near as rounding
    total = w.sum()
    for target in {p * total * (1 - 1e-12), p * total, p * total * (1 + 1e-12)} if p < 1 else {math.inf}:
        keep = (before < target) & (w >= min(m, 1.0))
        keep[0] = True
        stay = np.sort(first[keep])
        with np.errstate(over="ignore"):
            c = np.cumsum(np.exp((v[stay] - top) / heat))
        low, high = (min(int(np.searchsorted(c, (u + off) * c[-1], side="right")), len(stay) - 1) for off in (-1e-9, 1e-9))
        right.update(stay[low:high + 1].tolist())
    return right, {t: logp(t) for t in right}
