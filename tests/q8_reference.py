"""The 8-bit cache written out in numpy from the text of include/nsn.h: format, append, attention, eviction (64 bits, but for
the scales and their inverses, which the format defines in fp32)."""
from __future__ import annotations

import math

import numpy as np

F32 = np.float32
INT8, E4M3 = 0, 1


def e4m3_value(u):
    u = np.asarray(u, dtype=np.int64)
    e, f = (u >> 3) & 15, (u & 7).astype(np.float64)
    x = np.where(e > 0, (8 + f) * np.exp2(e - 10.0), f * 2.0 ** -9)
    x = np.where((u & 127) == 127, np.nan, x)
    return np.where(u >= 128, -x, x)


_E4M3 = e4m3_value(np.arange(127))   # 0 .. 448, ascending


def round_code(code, y):
    """Nearest code (ties to even) to y, as a number."""
    y = np.where(np.isnan(y), 0.0, np.asarray(y, dtype=np.float64))
    if code == INT8:
        return np.clip(np.rint(y), -127, 127)
    a = np.minimum(np.abs(y), 448.0)
    hi = np.searchsorted(_E4M3, a)               # _E4M3[hi] >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _E4M3[lo], _E4M3[hi] - a
    at = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(_E4M3[at], y)


def to_bytes(code, c):
    if code == INT8:
        return c.astype(np.int8).view(np.uint8)
    u = np.searchsorted(_E4M3, np.abs(c)).astype(np.uint8)
    return np.where(np.signbit(c), u | 128, u).astype(np.uint8)


def from_bytes(code, u):
    return u.view(np.int8).astype(np.float64) if code == INT8 else e4m3_value(u)


def level(code, amax):
    """Scale (fp32) of a block of largest magnitude amax."""
    if not amax >= 2.0 ** -117:
        return F32(0)
    if code == INT8:
        return F32(amax) / F32(127)
    e = math.frexp(amax / 448)
    return F32(2.0 ** (e[1] - 1 if e[0] == 0.5 else e[1]))


def offsets(kind, D, tokens):
    """Byte offset of (token, channel) inside a unit."""
    t, c = np.arange(tokens)[:, None], np.arange(D)[None, :]
    if kind == "k":
        return t * D + c
    n, m = 256 // D, D // 16
    return t // n * 256 + c // m * 16 + t % n * m + c % m


class Unit:
    """Codes (as numbers, NaN where a byte is no number) and scales of one head of one sequence."""

    def __init__(self, code, D, max_len):
        self.code, self.D, self.n = code, D, max_len
        self.c = np.zeros((max_len, D))
        self.s = np.zeros(max_len // 64, dtype=F32)

    def append(self, start, x):
        """x: fp64 [n][D] of 16-bit values."""
        x = x[:max(0, self.n - start)]
        if not len(x):
            return
        end = start + len(x)
        for blk in range(start // 64, -(-end // 64)):
            lo, hi = max(start, 64 * blk), min(end, 64 * blk + 64)
            new = x[lo - start:hi - start]
            finite = np.abs(new[np.isfinite(new)])
            asked = level(self.code, finite.max() if finite.size else 0.0)
            old = self.s[blk] if lo > 64 * blk else F32(0)
            lv = max(asked, old)
            if asked > old and lo > 64 * blk:
                at = slice(64 * blk, lo)
                self.c[at] = round_code(self.code, self.c[at].astype(F32) * F32(old / lv))
            inv = F32(1) / lv if lv > 0 else F32(0)
            with np.errstate(invalid="ignore"):
                y = new.astype(F32) * inv
            self.c[lo:hi] = round_code(self.code, y)
            self.s[blk] = lv

    def rows(self, n):
        return self.c[:n] * np.repeat(self.s.astype(np.float64), 64)[:n, None]


def attention(q, k, v, scale, vis):
    """q [R][D], k, v [n][D], vis [R]: tokens each row sees (or a truth table [R][n]).  (out, lse, p, sum p |v|)."""
    s = scale * (q @ k.T)
    seen = np.arange(k.shape[0])[None, :] < vis[:, None] if vis.ndim == 1 else vis
    s = np.where(seen, s, -np.inf)
    m = s.max(axis=1, initial=-np.inf)
    p = np.exp(s - np.where(np.isfinite(m), m, 0.0)[:, None])
    l = p.sum(axis=1)
    with np.errstate(divide="ignore"):
        lse = np.where(l > 0, m + np.log(l), -np.inf)
    p /= np.where(l > 0, l, 1.0)[:, None]
    return p @ v, lse, p, p @ np.abs(v)


def keep_of(w, n, keep, first, recent):
    """Ascending indices that stay of the n tokens with weights w."""
    if n <= keep:
        return np.arange(n)
    nan = np.isnan(w[:n])
    w = np.where(nan, -np.inf, w[:n].astype(np.float64))
    sure = (np.arange(n) < first) | (np.arange(n) >= n - recent)
    order = np.lexsort((np.arange(n), np.where(nan, 1, 0), -w, ~sure))
    return np.sort(order[:keep])
