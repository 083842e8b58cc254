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
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1).astype(np.int64)
    with np.errstate(all="ignore"):
        v = VALUES[c & 7] * np.where(c & 8, -1.0, 1.0) * np.repeat(scale_value(scales), 16, -1)
        return v.astype(np.float16).astype(np.float64)


def quantise(x):
    """(values, scale codes) of x [..., d]; a group that is not all finite is NaN."""
    g = x.reshape(*x.shape[:-1], -1, 16)
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
