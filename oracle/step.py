"""The server's update in plain numpy -- TEST INFRASTRUCTURE ONLY, like the rest of this package.

Gradient norm, AdamW and the 8-bit states, from their definitions: once operation by operation in float32 (what a state
must be bit for bit) and once in float64 (what a result must be near to).
"""
from __future__ import annotations

import numpy as np

BLOCK = 256
F = np.float32

# magnitudes of the e4m3 codes 0 .. 126: field 0 holds k/8 * 2^-6, field f the numbers (1 + k/8) * 2^(f - 7)
E4M3 = np.array([(k & 7) / 8.0 * 2.0 ** -6 if k < 8 else (1 + (k & 7) / 8.0) * 2.0 ** ((k >> 3) - 7) for k in range(127)])


def norm(grads, grad_scale=1.0, max_norm=np.inf):
    """(norm, factor) in float64 of a list of arrays."""
    s = sum(float(np.sum(np.square(g.astype(np.float64)))) for g in grads)
    if not np.isfinite(s):
        return grad_scale * np.sqrt(s), -1.0
    n = grad_scale * np.sqrt(s)
    return n, grad_scale * min(1.0, max_norm / (n + 1e-6))


def moments32(m, v, g, factor, b1, b2):
    with np.errstate(all="ignore"):
        g = g.astype(F) * F(factor)
        m = F(b1) * m + F(1.0 - b1) * g
        v = F(b2) * v + F(1.0 - b2) * (g * g)
    return m, v


def weight64(p, m, v, t, lr, b1, b2, eps, wd, root=None):
    """New weight and the two parts of its change, in float64, from the new moments."""
    p, m = p.astype(np.float64), m.astype(np.float64)
    root = np.sqrt(v.astype(np.float64)) if root is None else root.astype(np.float64)
    decay = lr * wd * p
    step = lr / (1.0 - b1 ** t) * (m / (root / np.sqrt(1.0 - b2 ** t) + eps))
    return p - (decay + step), decay, step


def _fin(x):
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(13))
    x = (x * np.uint64(0xBB67AE85)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random16(first, n, seed, t):
    """The 16 bits of the places first .. first + n - 1."""
    u = lambda x: np.uint64(x & 0xFFFFFFFF)  # noqa: E731
    k = _fin(u(int(t & 0xFFFFFFFF) * 0x9E3779B9 + 0x3C6EF372))
    k = _fin(u((seed >> 32) * 0x9E3779B9 + int(k)))
    k = _fin(u((seed & 0xFFFFFFFF) * 0x9E3779B9 + int(k)))
    place = np.arange(first, first + n, dtype=np.uint64)
    h = _fin((((place >> np.uint64(1)) & np.uint64(0xFFFFFFFF)) * np.uint64(0x9E3779B9) + k) & np.uint64(0xFFFFFFFF))
    return np.where(place & np.uint64(1), h >> np.uint64(16), h & np.uint64(0xFFFF)).astype(np.int64)


def decode(code, scale):
    """float32 values of whole blocks of codes (uint8) under their scales (uint8)."""
    s = np.repeat(scale.astype(np.int64), BLOCK)
    mag = np.append(E4M3, np.inf)[code & 127]        # 127 is no code that a state holds
    with np.errstate(over="ignore"):
        return np.where(code & 128, -1.0, 1.0).astype(F) * np.ldexp(mag, s - 127).astype(F)


def encode(x, r16, keep):
    """Codes and scales of whole blocks; ``keep``: what is not zero does not become zero."""
    a = np.abs(x.astype(np.float64)).reshape(-1, BLOCK)
    a = np.where(np.isnan(a), np.inf, a)
    top = a.max(axis=1)
    frac, ex = np.frexp(np.where(np.isfinite(top), top, 1.0))
    s = ex + 118 + (frac >= 0.875)                   # top = frac 2^ex stays within 448 = 0.875 * 2^9 of the scale 2^(s - 127)
    s = np.clip(np.where(top == 0.0, 0, s), 0, 247)
    s = np.where(np.isfinite(top), s, 247)
    y = np.ldexp(a, 127 - s[:, None]).reshape(-1)
    y = np.where(y < 2.0 ** -6, np.floor(np.ldexp(np.minimum(y, 1.0), 29)) * 2.0 ** -29, y)      # 20 bits below a code, here too
    lo = np.clip(np.searchsorted(E4M3, y, side="right") - 1, 0, 126)
    gap = np.append(np.diff(E4M3), np.inf)[lo]
    with np.errstate(invalid="ignore"):
        part = np.where(lo < 126, (y - E4M3[lo]) / gap, 0.0)
    cut = np.floor(np.where(np.isfinite(part), part, 0.0) * 2 ** 20).astype(np.int64)
    code = np.minimum(lo + (cut + 16 * r16 + 8 >= 2 ** 20), 126)
    if keep:
        code = np.where((y >= 0) & (x != 0), np.maximum(code, 1), code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8), s.astype(np.uint8)
