"""The operators of a worker's forward and backward pass by their definitions, in 64 bits on the CPU (NumPy), and the bounds that fp32
arithmetic keeps to.  Shares nothing with the library but the checkpoint's layout, which is its interface."""
import math

import numpy as np

EPS = 2.0 ** -24        # half a unit in the last place of fp32
GROUP = 32


def bf16(v):
    """v (float64 or float32 array) rounded to bfloat16, as float32."""
    v = np.asarray(v, np.float32)
    b = v.view(np.uint32).astype(np.uint64)
    r = ((b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(v), r, v)


def e4m3_values():
    """What the 256 codes stand for."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if e == 15 and m == 7 else math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        out[c] = -v if c & 128 else v
    return out


CODES = e4m3_values()


def scale_bytes(top):
    """Scale byte of each group's largest magnitude."""
    top = np.asarray(top, np.float64)
    out = np.empty(top.shape, np.uint8)
    for at in np.ndindex(top.shape):
        t = float(top[at])
        if not math.isfinite(t):
            out[at] = 255
            continue
        e = -117
        while t > 448.0 * 2.0 ** e and e < 119:
            e += 1
        out[at] = e + 127
    return out


def to_codes(v, byte):
    """E4M3 codes of v / 2^(byte - 127), nearest even, held to 448; v float64 [..][32], byte [..]."""
    q = np.clip(v * 2.0 ** -(byte[..., None].astype(np.float64) - 127), -448.0, 448.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6))) - 3)
    r = np.abs(np.rint(q / step) * step)
    e = np.floor(np.log2(np.maximum(r, 2.0 ** -6)))
    low = r < 2.0 ** -6
    code = np.where(low, r * 2.0 ** 9, (e + 7) * 8 + (r / 2.0 ** e - 1) * 8).astype(np.uint8)
    return code | (np.signbit(v) * 128).astype(np.uint8)


def groups_of(v):
    """[rows][G][32], zeros behind the rows' ends."""
    rows, n = v.shape
    g = -(-n // GROUP)
    out = np.zeros((rows, g * GROUP))
    out[:, :n] = v
    return out.reshape(rows, g, GROUP)


def encode(v):
    """(codes [rows][G * 32], scales [rows][G]) of a float64 matrix that holds fp32 numbers."""
    t = groups_of(v)
    bad = ~np.isfinite(t).all(-1)
    byte = scale_bytes(np.where(bad, np.inf, np.abs(np.where(np.isfinite(t), t, 0)).max(-1)))
    codes = to_codes(np.where(bad[..., None], 0.0, t), np.where(bad, 127, byte).astype(np.uint8))
    inside = groups_of(np.ones(v.shape)) > 0
    codes = np.where(inside, np.where(bad[..., None], 0x7f, codes), 0).astype(np.uint8)
    return codes.reshape(v.shape[0], -1), byte


def decode(codes, scales, n):
    """float64 [rows][n]."""
    e = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (CODES[codes].reshape(scales.shape + (GROUP,)) * e[..., None]).reshape(codes.shape)[:, :n]


def norm_forward(x, residual, weight, eps):
    v = x if residual is None else x + residual
    rstd = 1.0 / np.sqrt((v * v).mean(1) + eps)
    xhat = v * rstd[:, None]
    return v, rstd, xhat, xhat if weight is None else xhat * weight


def norm_backward(dy, xhat, rstd, weight, dh):
    """dx, dweight, and the bounds of what fp32 sums (at most 80 additions one after the other over a row, 200 over the rows) may be off."""
    g = dy if weight is None else dy * weight
    n = dy.shape[1]
    c = (g * xhat).sum(1, keepdims=True) / n
    dx = rstd[:, None] * (g - xhat * c)
    size = np.abs(g * xhat).sum(1, keepdims=True) / n
    off = np.abs(rstd)[:, None] * (4 * np.abs(g) + np.abs(xhat) * (90 * size + 4 * np.abs(c))) * EPS
    if dh is not None:
        dx = dx + dh
        off = off + np.abs(dh) * EPS
    return dx, off + np.abs(dx) * 2 * EPS, (dy * xhat).sum(0), 210 * EPS * np.abs(dy * xhat).sum(0)


def policy(logits, tokens, old, ref, adv, weight, low, high, kl):
    """logp, losses, dlogits and how far fp32 may be off each; float64 arrays, None where not given."""
    rows, n = logits.shape
    logp, losses, grad = np.zeros(rows), np.zeros(rows), np.zeros((rows, n))
    off = np.zeros(rows), np.zeros(rows), np.zeros((rows, n))
    tol = (n / 1024 + 120) * EPS            # of the sum: additions one after the other, exponentials
    for t in range(rows):
        q = 1.0 if weight is None else weight[t]
        a = int(tokens[t])
        if q == 0 or not 0 <= a < n:
            continue
        top = logits[t].max()
        with np.errstate(invalid="ignore"):
            e = np.exp(logits[t] - top)
        s = e.sum()
        with np.errstate(invalid="ignore"):
            logp[t] = logits[t, a] - top - math.log(s)
            # exponents are off by their own rounding: of the terms that weigh, a few tens at most
            off[0][t] = tol + 4 * EPS * (abs(logits[t, a] - top) + math.log(s) + 16)
        if adv is None:
            continue
        r = 1.0 if old is None else math.exp(logp[t] - old[t])
        held = min(max(r, 1 - low), 1 + high)
        f, c = -min(r * adv[t], held * adv[t]), -adv[t] * r if r * adv[t] <= held * adv[t] else 0.0
        d_tol = off[0][t] + (0 if old is None else 2 * EPS * (abs(logp[t]) + abs(old[t])))
        f_off = abs(adv[t]) * r * (0 if old is None else d_tol) + abs(f) * 4 * EPS
        c_off = f_off
        if ref is not None:
            d = ref[t] - logp[t]
            m = math.expm1(d)
            f += kl * (m - d)
            c -= kl * m
            k_off = off[0][t] + 2 * EPS * (abs(logp[t]) + abs(ref[t]))
            f_off += kl * (abs(m) * k_off + 4 * EPS * (abs(m) + abs(d)) + k_off * k_off)
            c_off += kl * ((abs(m) + 1) * k_off + 4 * EPS * abs(m))
        losses[t], off[1][t] = q * f, abs(q) * (f_off + 4 * EPS * abs(f))
        p = e / s
        one = np.zeros(n)
        one[a] = 1.0
        grad[t] = q * c * (one - p)
        with np.errstate(invalid="ignore"):
            x_off = np.where(p > 0, 4 * EPS * np.abs(logits[t] - top), 0.0)
        off[2][t] = abs(q) * ((one + p) * (c_off + 8 * EPS * abs(c)) + abs(c) * p * (tol + x_off)) + 1e-37
    return logp, losses, grad, off
