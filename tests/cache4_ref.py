"""4-bit pages in 64 bits (numpy), for the tests."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
NAN_SCALE = 0xff


def scale_value(code):
    """The scale of a byte: 5 exponent bits (bias 15), 3 mantissa bits; exponent 31 is not finite."""
    code = code.astype(np.int64)
    e, m = code >> 3, (code & 7).astype(np.float64)
    v = np.where(e > 0, (8 + m) * np.exp2(np.where(e < 31, e, 0) - 18.0), m * 2.0 ** -17)
    return np.where(e == 31, np.where(m == 0, np.inf, np.nan), v)


def scale_code(a):
    """The byte of max / 6 = a: to the nearest scale, ties to even, 10240 at most."""
    a = np.asarray(a, np.float64)
    unit = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -14))) - 3)
    v = np.minimum(np.round(a / unit) * unit, 10240.0)
    e = np.floor(np.log2(np.maximum(v, 2.0 ** -14)))
    return np.where(v >= 2.0 ** -14, (e + 14) * 8 + v / np.exp2(e - 3), v * 2.0 ** 17).astype(np.uint8)


def nearest(x):
    """x to the nearest value of a code, ties to the even code, 6 at most."""
    m = np.abs(x)
    step = np.where(m < 2, 0.5, np.where(m < 4, 1.0, 2.0))
    return np.sign(x) * np.minimum(np.round(m / step) * step, 6)


def decode(codes, scales):
    """Values [..., d] of codes [..., d / 2] with scales [..., d / 16], in f16 as the kernels form them."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1]).astype(np.int64)
    with np.errstate(all="ignore"):
        v = VALUES[c & 7] * np.where(c & 8, -1.0, 1.0) * np.repeat(scale_value(scales), 16, -1)
        return v.astype(np.float16).astype(np.float64)


def quantise(x):
    """(values, scale codes) of x [..., d]; a group that is not all finite is NaN."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0)
    code = scale_code(np.abs(g).max(-1) / 6)
    s = scale_value(code)[..., None]
    v = np.where(s > 0, nearest(g / np.where(s > 0, s, 1)) * s, 0)
    return np.where(fine[..., None], v, np.nan).reshape(x.shape), np.where(fine, code, NAN_SCALE).astype(np.uint8)


def check_quantised(values, scales, x, err):
    """That `values` [..., d] with scale bytes [..., d / 16] are what some x' with |x' - x| <= err rounds to: rounding
    is monotonic, so the scale and then each code lie between those of the ends."""
    g, e = x.reshape(*x.shape[:-1], -1, 16), err.reshape(*x.shape[:-1], -1, 16)
    low, high = np.maximum(np.abs(g) - e, 0).max(-1), (np.abs(g) + e).max(-1)
    u = 2.0 ** -24   # of the division by 6, and of that by the scale
    assert (scale_code(low / 6 * (1 - u)) <= scales).all() and (scales <= scale_code(high / 6 * (1 + u))).all()
    s = scale_value(scales)[..., None]
    d = np.where(s > 0, s, 1)
    lo, hi = nearest((g - e) / d * np.where(g > e, 1 - u, 1 + u)) * s, nearest((g + e) / d * np.where(g < -e, 1 - u, 1 + u)) * s
    v = values.reshape(g.shape)
    assert (np.minimum(lo, hi) <= v).all() and (v <= np.maximum(lo, hi)).all()


def attention(q, k, v, length, causal=True, window=0, sinks=0, scale=None):
    """One sequence: q [n, H_q, d], k, v [length, H, d] f64 -> (o, lse, bound of o before its rounding, bound of lse)."""
    U32 = 2.0 ** -24
    n, Hq, d = q.shape
    H = k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    p, j = length - n + np.arange(n)[:, None], np.arange(length)[None, :]
    see = np.ones((n, length), bool)
    if causal:
        see &= j <= p
    if window > 0:
        see &= (j > p - window) | (j < sinks)
    see &= p >= 0 if causal else True
    o, eo = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, el = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    seen = see.any(0)[:, None]
    for h in range(Hq):
        kk, vv = np.where(seen, k[:, h // (Hq // H)], 0), np.where(seen, v[:, h // (Hq // H)], 0)
        x = np.where(see, q[:, h] @ kk.T * scale, -np.inf)
        size = np.where(see, np.abs(q[:, h]) @ np.abs(kk).T * abs(scale), 0)
        top = x.max(1, initial=-np.inf, keepdims=True)
        w = np.where(see, np.exp(x - np.where(np.isfinite(top), top, 0)), 0)
        s = w.sum(1, keepdims=True)
        some = s[:, 0] > 0
        prob = np.divide(w, s, out=np.zeros_like(w), where=s > 0)
        o[:, h] = prob @ vv
        lse[some, h] = (top + np.log(np.where(s > 0, s, 1)))[some, 0]
        # a logit is off by at most (d + 8) u32 of its absolute sum (an f32 sum in any order) and by the scale's and the
        # exponent's rounding; a probability is an f16 number: 2^-11 of itself, or 2^-32 of the row's largest
        logit = (d + 8) * U32 * size.max(1, initial=0) + 4 * U32 * np.abs(np.where(see, x, 0)).max(1, initial=0)
        eo[:, h] = (2.0 ** -11 + 2 * logit[:, None] + length * U32 + 2.0 ** -20) * (prob @ np.abs(vv)) + 2.0 ** -32 * (see @ np.abs(vv))
        el[:, h] = logit + length * U32 + 2.0 ** -20 * (1 + np.abs(np.where(some, lse[:, h], 0)))
    return o, lse, eo, el
