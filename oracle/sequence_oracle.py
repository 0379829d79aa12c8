"""Plain numpy implementations in 64 bits of the operators for training recurrent sequence models: linear attention with a
decay for each head and its gradients, step by step; the clipped policy loss with its gradient; AdamW with states in 32 and in 8 bits.
Written from the formulas, slow on purpose; shares no code with the CUDA library."""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ linear attention (one sequence and head)
def linear_attention(q, k, v, log_decay, scale=1.0, S0=None):
    """o [n, Dv] and the last state: S = lambda S + k v^T, o = scale S^T q."""
    lam = np.exp(np.float64(log_decay))
    S = np.zeros((k.shape[1], v.shape[1])) if S0 is None else np.array(S0, np.float64)
    o = np.zeros((q.shape[0], v.shape[1]))
    for t in range(q.shape[0]):
        S = lam * S + np.outer(k[t], v[t])
        o[t] = scale * (S.T @ q[t])
    return o, S


def linear_attention_backward(q, k, v, log_decay, do, scale=1.0, S0=None, dS=None):
    """dq, dk, dv, dS0."""
    lam = np.exp(np.float64(log_decay))
    n, Dk, Dv = q.shape[0], k.shape[1], v.shape[1]
    states, S = [], np.zeros((Dk, Dv)) if S0 is None else np.array(S0, np.float64)
    for t in range(n):
        S = lam * S + np.outer(k[t], v[t])
        states.append(S)
    R = np.zeros((Dk, Dv)) if dS is None else np.array(dS, np.float64)       # d loss / d S_t
    dq, dk, dv = np.zeros((n, Dk)), np.zeros((n, Dk)), np.zeros((n, Dv))
    for t in range(n - 1, -1, -1):
        dq[t] = scale * (states[t] @ do[t])
        R = R + scale * np.outer(q[t], do[t])
        dk[t], dv[t] = R @ v[t], R.T @ k[t]
        R = lam * R
    return dq, dk, dv, R


# ------------------------------------------------------------------ policy loss (one row)
def policy_loss(z, action, old, adv, w, ref=None, clip_low=0.2, clip_high=0.2, kl=0.0):
    """loss, logp, dz of one row."""
    z = np.asarray(z, np.float64)
    with np.errstate(all="ignore"):
        top = z.max()
        lse = top + np.log(np.sum(np.exp(z - top)))
        logp = z[action] - lse if 0 <= action < len(z) else np.nan
        if w == 0:
            return 0.0, logp, np.zeros_like(z)
        r = np.exp(logp - old)
        free, held = r * adv, np.clip(r, 1 - clip_low, 1 + clip_high) * adv
        loss, g = -min(free, held), (-free if free <= held else 0.0)
        if ref is not None:
            d = ref - logp
            loss, g = loss + kl * (np.expm1(d) - d), g - kl * np.expm1(d)
        p = np.exp(z - lse)
        one = np.zeros_like(z)
        if 0 <= action < len(z):
            one[action] = 1
        if np.isnan(logp):
            return np.nan, np.nan, np.full_like(z, np.nan)
        return w * loss, logp, w * g * (one - p)


# ------------------------------------------------------------------ AdamW
def adamw(p, g, m, v, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=1.0):
    """New p, m, v in 64 bits."""
    b1, b2 = betas
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    g = g * grad_scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = p * (1 - lr * weight_decay) - lr * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p, m, v


def adamw_f32(p, g, m, v, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None):
    """The step in fp32, one rounding an operation, in the documented order; also sqrt(v)."""
    f = np.float32
    b1, b2 = betas
    g = np.asarray(g, f)
    if grad_scale is not None:
        g = g * f(grad_scale)
    m = m * f(b1) + g * f(1 - b1)
    v = v * f(b2) + (g * g) * f(1 - b2)
    root = np.sqrt(v)
    p = p * f(1 - lr * weight_decay) - (m * f(lr / (1 - b1 ** step))) / (root * f(1 / np.sqrt(1 - b2 ** step)) + f(eps))
    return p, m, v, root


def random_bits(place, seed):
    """32 random bits of a state's place."""
    out = []
    for n in np.asarray(place, dtype=object).reshape(-1):
        w = 0xFFFFFFFF
        x = ((int(n) & w) + seed * 0x6A09E667 + (int(n) >> 32) * 0xBB67AE85) & w
        x = (x ^ (x >> 16)) * 0x6A09E667 & w
        x = (x ^ (x >> 15)) * 0xBB67AE85 & w
        x = (x ^ (x >> 16)) * 0x3C6EF373 & w
        out.append(x ^ (x >> 15))
    return np.array(out, np.uint64)


def float8_value(code):
    """Value of an 8-bit float: sign, 4 exponent bits (bias 7), 3 mantissa bits."""
    code = np.asarray(code, np.int64)
    e, f, s = (code >> 3) & 15, code & 7, np.where(code & 128, -1.0, 1.0)
    x = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e.astype(np.float64) - 7))
    return np.where((code & 127) == 127, np.nan, s * x)


def float8_cut(x, random16):
    """Codes and scale of one block of fp32 values: scale a power of two, every value rounded by its 16 random bits."""
    x = np.asarray(x, np.float32)
    big = np.abs(x).max()
    scale = max(2.0 ** (np.floor(np.log2(np.float64(big))) - 7), 2.0 ** -120) if big > 0 else 2.0 ** -120
    codes = []
    for v, r in zip(x, random16):
        a = np.float32(abs(np.float64(v)) / scale)
        r = int(r)
        if a >= 2.0 ** -6:
            bits = int(a.view(np.uint32)) + r * 16
            c = (bits >> 20) - 120 * 8
        else:
            c = int(np.floor(np.float32(np.float32(a * np.float32(512)) + np.float32(r * 2.0 ** -16))))
        codes.append(c | (128 if np.signbit(v) else 0))
    return np.array(codes, np.uint8), np.float32(scale)
