"""Plain models that the tests of a generating step compare with: drawn tokens in whole numbers, residual sums with
their norms in 64 bits, and what an 8-bit cache holds."""
import math

import numpy as np

COEFFICIENTS = [-0.00089964044, 0.0090985559, -0.055210155, 0.24015228, -0.69314098, 1.0]


def weights(x, scale):
    """Whole-number weights of one row's logits (float32), and their distances t."""
    x = np.asarray(x, np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        t = ((x.max() - x) * (np.float32(scale) * np.float32(1.44269504088896340736))).astype(np.float32)
    t = np.minimum(np.where(np.isnan(t), np.float32(63), t), np.float32(63))
    n = np.floor(t)
    f = (t - n).astype(np.longdouble)
    p = np.full(x.shape, COEFFICIENTS[0], np.float32)
    for c in COEFFICIENTS[1:]:  # fused: the product is exact, the sum nearly
        p = (p.astype(np.longdouble) * f + np.longdouble(np.float32(c))).astype(np.float32)
    assert p.min() >= 0.5 and p.max() <= 1.0
    return (p.astype(np.float64) * 2.0**24).astype(np.int64) << 16 >> n.astype(np.int64), t


def sample(x, u, top_k, top_p, min_p, scale):
    """One row: id, log probability, tokens kept."""
    x = np.asarray(x, np.float32)
    if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all() or not 0 <= u < 1:
        return -1, math.nan, 0
    w, t = weights(x, scale)
    order = np.argsort(-x, kind="stable")
    sums = w[order]
    if top_k:
        sums = sums[:top_k]
    keep = len(sums)
    before = np.cumsum(sums) - sums
    if top_p < 1:
        keep = int((before < math.ceil(float(sums.sum()) * float(np.float32(top_p)))).sum())
    kept = np.zeros(len(x), bool)
    kept[order[:keep]] = True
    if min_p > 0:
        kept &= t <= np.float32(-math.log2(float(np.float32(min_p))))
    kept &= w > 0
    w = np.where(kept, w, 0)
    total = int(w.sum())
    place = (int(float(np.float32(u)) * 2.0**31) * total) >> 31
    i = int(np.searchsorted(np.cumsum(w), place, side="right"))
    return i, -(float(t[i]) * math.log(2) + math.log1p((total - 2**40) / 2**40)), int(kept.sum())


def norm(x, weight, y, out_weight, gate, scale, eps):
    """s and its norm (None without weight), rows in float64."""
    rms = lambda a: np.sqrt((a * a).mean(1, keepdims=True) + eps)
    s = x
    if y is not None:
        z = y if out_weight is None else y / rms(y) * out_weight
        s = x + scale * (z if gate is None else gate * z)
    return s, None if weight is None else s / rms(s) * weight


def stored(x):
    """What an 8-bit cache holds of rows x [..., d] of finite values or not: values, codes and exponents' bytes."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    most = np.where(fine, np.abs(x), 0).max(-1, keepdims=True)
    m, p = np.frexp(most)  # most = m 2^p, m in [1/2, 1): 448 = 0.875 2^9
    e = np.where(most > 0, np.maximum(p - 9 + (m > 0.875), -126), -126)
    c = np.where(fine, x, 0) / 2.0**e
    power = np.maximum(np.frexp(c)[1] - 1, -6)
    c = np.rint(c / 2.0**(power - 3)) * 2.0**(power - 3)  # to even
    power = np.maximum(np.frexp(c)[1] - 1, -6)
    low = c == 0
    mantissa = np.abs(c) / 2.0**(power - 3)  # 8 .. 15, or less below 2^-6
    code = np.where(mantissa >= 8, (power + 7) * 8 + mantissa - 8, mantissa).astype(np.int64)
    sign = np.signbit(np.where(fine, x, 0))
    code = np.where(low, 0, code) | sign.astype(np.int64) << 7
    values = np.where(fine, c * 2.0**e, np.nan)
    return values, np.where(fine, code, -1), (e[..., 0] + 127).astype(np.int64)


def held(codes, powers):
    """The values of an 8-bit cache's codes [..., d] and bytes [...]."""
    codes = np.asarray(codes, np.int64)
    low, power = codes & 7, codes >> 3 & 15
    size = np.where(power > 0, (1 + low / 8) * 2.0**(power - 7), low * 2.0**-9)
    size = np.where((codes & 127) == 127, np.nan, size)
    return np.where(codes >> 7, -size, size) * 2.0**(np.asarray(powers, np.float64)[..., None] - 127)
