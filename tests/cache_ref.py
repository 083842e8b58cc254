"""The paged KV cache's operators in 64 bits (numpy), for the tests: rotary positions, the append and
the attention, with the bounds that their kernels' rounding allows."""
from __future__ import annotations

import numpy as np

U32, UBF = 2.0 ** -24, 2.0 ** -8      # unit roundoff of f32 and bf16


def frequencies(rot, base=10000.0, sections=None, scaling=None):
    """Radians a position of each pair, its axis, and the amplitude."""
    f, axis, amp = [], [], 1.0
    for a, n in enumerate(sections or [rot // 2]):
        for k in range(n):
            b = base
            if scaling and scaling[0] == "stretch":
                b = base * scaling[1] ** (n / (n - 1.0))
            w = b ** (-k / n)
            if scaling and scaling[0] == "linear":
                w = w / scaling[1]
            if scaling and scaling[0] == "parts":
                turns = scaling[2] * w / (2 * np.pi)
                keep = np.clip((turns - 1) / 31, 0, 1)
                w = w * (keep + (1 - keep) / scaling[1])
                amp = 1 + 0.1 * np.log(scaling[1])
            f.append(w)
            axis.append(a)
    return np.array(f), np.array(axis), amp


def rotate(x, positions, rot, layout="half", inverse=False, **kw):
    """x [T, H, d] f64 by integer positions [T, axes] -> (rotated, bound of an f32 computation)."""
    f, axis, amp = frequencies(rot, **kw)
    n = rot // 2
    lo, hi = (np.arange(n), np.arange(n) + n) if layout == "half" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    angle = positions[:, axis].astype(np.float64) * f * (-1 if inverse else 1)
    c, s = np.cos(angle)[:, None] * amp, np.sin(angle)[:, None] * amp
    y, err = x.copy(), np.zeros_like(x)
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    # the angle's rounding (pi u), the sine's and cosine's (2 ulp = 4 u), amplitude, product, sum
    e = 11 * U32 * amp * (np.abs(a) + np.abs(b)) + 1e-12 * (np.abs(a) + np.abs(b)) * np.abs(angle).max(initial=0)
    err[..., lo], err[..., hi] = e, e
    return y, err


def e4m3(x):
    """x to the nearest e4m3 value, ties to even (|x| <= 448)."""
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.round(x / step) * step


def e4m3_step(x):
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)


def page_scale(amax):
    """Least power of two with amax <= 448 times it, between 2^-120 and 2^120."""
    if amax <= 0:
        return 2.0 ** -120
    e = int(np.ceil(np.log2(amax / 448)))
    while 448 * 2.0 ** e < amax:
        e += 1
    while amax <= 448 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** min(max(e, -120), 120)


def attention(q, k, v, n_new, length, causal=True, window=0, sinks=0, scale=None):
    """One sequence: q [n_new, H_q, d], k, v [length, H, d] f64 -> (o, lse, bound of o, bound of lse)."""
    T, Hq, d = q.shape
    L, H = k.shape[0], k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    p = length - n_new + np.arange(T)[:, None]
    j = np.arange(L)[None, :]
    see = np.ones((T, L), bool)
    if causal:
        see &= j <= p
    if window > 0:
        see &= (j > p - window) | (j < sinks)
    o, eo = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    lse, el = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for h in range(Hq):
        kk, vv = np.where(see.any(0)[:, None], k[:, h // (Hq // H)], 0), np.where(see.any(0)[:, None], v[:, h // (Hq // H)], 0)
        x = np.where(see, q[:, h] @ kk.T * scale, -np.inf)
        size = np.where(see, np.abs(q[:, h]) @ np.abs(kk).T * abs(scale), 0)
        top = x.max(1, initial=-np.inf, keepdims=True)
        w = np.where(see, np.exp(x - np.where(np.isfinite(top), top, 0)), 0)
        s = w.sum(1, keepdims=True)
        some = s[:, 0] > 0
        prob = np.divide(w, s, out=np.zeros_like(w), where=s > 0)
        o[:, h] = prob @ vv
        lse[some, h] = (top + np.log(np.where(s > 0, s, 1)))[some, 0]
        # a logit is off by at most (d + 8) u32 of its absolute sum (an f32 sum in any order), and by
        # the scale's and the exponent's rounding; a probability is rounded to bf16 before the product
        logit = (d + 8) * U32 * size.max(1, initial=0) + 4 * U32 * np.abs(np.where(see, x, 0)).max(1, initial=0)
        part = prob @ np.abs(vv)
        eo[:, h] = (UBF + 2 * logit[:, None] + L * U32 + 2.0 ** -20) * part + UBF * np.abs(o[:, h])
        el[:, h] = logit + L * U32 + 2.0 ** -20 * (1 + np.abs(np.where(some, lse[:, h], 0)))
    return o, lse, eo, el
