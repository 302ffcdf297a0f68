"""Plain definitions in 64 bits of the operators around a feed-forward block's products (TEST INFRASTRUCTURE ONLY): norm, the 8-bit
format, gated projections, and their gradients.  numpy alone; nothing is shared with the GPU library.  Inputs are float64 arrays that hold bf16 values.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def bf16_round(x):
    """Each value of a float64 array rounded to bf16 (8 significant bits, ties to even; the exponent range of fp32, subnormals included)."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    fine = np.isfinite(x) & (x != 0)
    e = np.maximum(np.frexp(x[fine])[1] - 1, -126)
    step = np.ldexp(1.0, e - 7)
    r = np.round(x[fine] / step) * step
    r[np.abs(r) >= 2.0 ** 128] = np.copysign(np.inf, r[np.abs(r) >= 2.0 ** 128])
    out[fine] = r
    return out


# ---- the 8-bit format -------------------------------------------------------------------------------------------------------


def e4m3_value(code):
    """What an e4m3 byte stands for: sign, four bits of exponent (bias 7), three of fraction; no infinities, 0x7F and 0xFF are NaN."""
    sign, exponent, fraction = code >> 7, code >> 3 & 15, code & 7
    if exponent == 15 and fraction == 7:
        return math.nan
    magnitude = math.ldexp(fraction, -9) if exponent == 0 else math.ldexp(8 + fraction, exponent - 10)
    return -magnitude if sign else magnitude


E4M3 = np.array([e4m3_value(c) for c in range(256)])


def e4m3_codes(x):
    """Bytes of the e4m3 values nearest to x (|x| <= 448), ties to the even fraction; NaN's byte without its sign."""
    x = np.asarray(x, dtype=np.float64)
    codes = np.full(x.shape, 0x7F, dtype=np.uint8)
    fine = np.isfinite(x)
    m = np.abs(x[fine])
    assert m.size == 0 or m.max() <= 448.0
    e = np.maximum(np.frexp(m)[1] - 1, -6)
    steps = np.round(np.ldexp(m, 3 - e)).astype(np.int64)   # in units of the last place; 16 carries into the next exponent
    code = np.where(steps < 8, steps, (e + 7) * 8 + steps - 8)
    codes[fine] = code + 128 * np.signbit(x[fine])
    return codes


def q8_exponents(x):
    """[rows, blocks]: the least e >= -127 with max|finite| <= 448 * 2^e of each block of 128 columns; 0 for a block of zeros."""
    rows, cols = x.shape
    n = -(-cols // BLOCK)
    v = np.zeros((rows, n * BLOCK))
    v[:, :cols] = np.where(np.isfinite(x), np.abs(x), 0.0)
    most = v.reshape(rows, n, BLOCK).max(2)
    e = np.full(most.shape, -127, dtype=np.int64)
    for k in range(-127, 128):   # as it is defined: the first that is large enough
        e = np.where((e == k) & (most > 448.0 * 2.0 ** k), k + 1, e)
    return np.where(most == 0, 0, e)


def q8_quantize(x):
    """(codes [rows, padded], exponents [rows, blocks]) of a matrix along its rows."""
    rows, cols = x.shape
    e = q8_exponents(x)
    v = np.zeros((rows, e.shape[1] * BLOCK))
    v[:, :cols] = x
    with np.errstate(invalid="ignore"):
        v = np.ldexp(v, -np.repeat(e, BLOCK, 1))
    return e4m3_codes(v), e


def q8_values(codes, e, cols):
    return np.ldexp(E4M3[codes], np.repeat(e, BLOCK, 1))[:, :cols]


def q8_rounded(x):
    return q8_values(*q8_quantize(x), x.shape[1])


# ---- norm -------------------------------------------------------------------------------------------------------------------


def rmsnorm(x, residual, weight, eps):
    """(sum, y, rstd)"""
    z = x if residual is None else x + residual
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt((z * z).mean(1) + eps)
        return z, z * rstd[:, None] * weight, rstd


def rmsnorm_bwd(dy, z, weight, rstd, dsum):
    """(dx, dweight)"""
    r = rstd[:, None]
    t = dy * weight
    dx = r * t - z * r ** 3 * (t * z).mean(1, keepdims=True)
    return dx if dsum is None else dx + dsum, (dy * z * r).sum(0)


# ---- gated projections ------------------------------------------------------------------------------------------------------

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activation(g, name):
    """(act(g), act'(g))"""
    if name == "silu":
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-g))
        return g * p, p + g * p * (1.0 - p)
    cdf = 0.5 * _erfc(-g / math.sqrt(2.0))   # 1 + erf has no digits left where g is far below zero
    return g * cdf, cdf + g * np.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)


def gated(x, w, name):
    """(h, gu) for w [D, 2F]"""
    gu = x @ w
    g, u = np.split(gu, 2, axis=1)
    return activation(g, name)[0] * u, gu


def gated_slopes(dh, gu, name):
    """(dgu, h)"""
    g, u = np.split(gu, 2, axis=1)
    a, slope = activation(g, name)
    return np.concatenate([dh * u * slope, dh * a], 1), a * u
