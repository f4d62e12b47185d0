"""Oracle of the AdamW step: the formulas in float64, and the 8-bit states to the bit.

    g' = k g      m = b1 m + (1 - b1) g'      v = b2 v + (1 - b2) g'^2
    w = w (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)

(decoupled weight decay, Loshchilov and Hutter).  8-bit states: 256 values share the exponent field E of their largest
magnitude as a float32; a value is held as the upper bits of the float32 |x| 2^(top - E), sign and seven bits with top = 14 for m,
eight bits with top = 30 for v, rounded by adding sixteen random bits below the last place that is kept.
"""
from __future__ import annotations

import numpy as np

GROUP, TOP_M, TOP_V = 256, 14, 30


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))


def step(w, g, m, v, lr, b1, b2, eps, decay, t, k=1.0):
    """(w, m, v) after the step, float64."""
    w, g, m, v = (np.asarray(a, np.float64) for a in (w, g, m, v))
    g = g * k
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return w * (1 - lr * decay) - lr / (1 - b1 ** t) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** t) + eps), m, v


def moments_f32(g, m, v, b1, b2, k=1.0):
    """(m, v) after the step as float32 arithmetic gives them, one rounded operation at a time."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = np.asarray(g, f) * f(k)
        return f(b1) * np.asarray(m, f) + f(1 - b1) * g, f(b2) * np.asarray(v, f) + f(1 - b2) * (g * g)


def dither(index, seed):
    """32 bits from the index of a value among the groups and the step's seed."""
    mask = np.uint64(0xFFFFFFFF)
    h = (np.asarray(index, np.uint64) + np.uint64(seed * 0x9E3779B1 & 0xFFFFFFFF)) & mask
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x243F6A89)) & mask
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0xB7E15163)) & mask
    return (h ^ (h >> np.uint64(16))).astype(np.uint32)


def _groups(x):
    out = np.zeros(-(-x.size // GROUP) * GROUP, x.dtype)
    out[:x.size] = x
    return out.reshape(-1, GROUP)


def encode(x, top, bits):
    """(codes, exponents) of the float32 values of one tensor; bits: 16 random ones for each value."""
    x = np.asarray(x, np.float32)
    mag = x.view(np.uint32) & np.uint32(0x7FFFFFFF)
    exp = _groups(mag).max(1) >> 23 if x.size else np.zeros(0, np.uint32)
    e = np.repeat(exp, GROUP)[:x.size].astype(np.int64)
    with np.errstate(all="ignore"):
        near = np.ldexp(mag.view(np.float32).astype(np.float64), top - e).astype(np.float32)
    code = (near.view(np.uint32).astype(np.uint64) + (np.asarray(bits, np.uint64) << np.uint64(4))) >> np.uint64(20)
    if top == TOP_V:
        code = np.where((mag > 0) & (code == 0), 1, code)
    else:
        code = code | (x.view(np.uint32) >> 31 << 7).astype(np.uint64)
    return np.where(e == 255, 0, code).astype(np.uint8), exp.astype(np.uint8)


def decode(code, exp, top):
    """The float32 values that codes stand for."""
    code = np.asarray(code, np.uint8)
    e = np.repeat(np.asarray(exp, np.int64), GROUP)[:code.size]
    keep = np.uint32(0x7F if top == TOP_M else 0xFF)
    near = ((code.astype(np.uint32) & keep) << np.uint32(20)).view(np.float32)
    x = np.ldexp(near.astype(np.float64), e - top).astype(np.float32)
    if top == TOP_M:
        x = np.where(code >= 128, -x, x)
    return np.where(e == 255, np.float32(np.nan), x).astype(np.float32)


def spacing(x, exp, top):
    """Distance of the two codes' values that x lies between (float64)."""
    x = np.abs(np.asarray(x, np.float64))
    lowest = np.repeat(np.asarray(exp, np.int64), GROUP)[:x.size] - top - 126       # exponent of the smallest normal code
    with np.errstate(divide="ignore"):
        place = np.where(x > 0, np.floor(np.log2(np.where(x > 0, x, 1))), -10 ** 6).astype(np.int64)
    return np.ldexp(1.0, np.maximum(place, lowest) - 3)
