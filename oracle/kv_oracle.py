"""Slow CPU oracle of the serving operators: block tables and slots of a step, the 8-bit cache of keys and values,
attention over it.  numpy, float64, one request, head and token at a time; written from the definitions in
include/glowq.h (cache format, order of pages, visible keys) and sharing nothing with the kernels."""
from __future__ import annotations

import math

import numpy as np

EXP_MIN = -64
NAN_CODE = 0x7F


def code_values() -> np.ndarray:
    """The value of every E4M3 code: sign, four exponent bits with bias 7, three fraction bits, no infinities."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if c & 127 == 127 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out[c] = -v if c & 128 else v
    return out


VALUES = code_values()
# (magnitudes 0 .. 448 in order of their codes; neighbours' midpoints decide, ties go to the even code)
MAGNITUDES = VALUES[:127]


def encode(x: np.ndarray) -> np.ndarray:
    """E4M3 codes of numbers of magnitude <= 448, nearest even; NaN code for what is not finite."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 1, 126)
    lo = hi - 1
    mid = (MAGNITUDES[lo] + MAGNITUDES[hi]) / 2
    code = np.where(a < mid, lo, np.where(a > mid, hi, np.where(lo % 2 == 0, lo, hi))).astype(np.uint8)
    code = np.where(a == 0, 0, code).astype(np.uint8)
    code = np.where(np.signbit(x), code | 128, code).astype(np.uint8)
    return np.where(np.isfinite(x), code, NAN_CODE).astype(np.uint8)


def exponent(top: float) -> int:
    """The smallest e >= EXP_MIN with top <= 448 * 2^e."""
    e = EXP_MIN
    while top > math.ldexp(448.0, e):
        e += 1
    return e


def key_byte(t: int, d: int, D: int) -> int:
    return ((t // 16) * (D // 64) + d // 64) * 1024 + ((d % 64) // 16) * 256 + (t % 16) * 16 + d % 16


def value_byte(t: int, d: int, D: int) -> int:
    return ((t // 16) * (D // 64) + d // 64) * 1024 + ((t % 16) // 4) * 256 + (d % 16) * 16 + ((d % 64) // 16) * 4 + t % 4


def places(B: int, D: int, values: bool) -> np.ndarray:
    f = value_byte if values else key_byte
    return np.array([[f(t, d, D) for d in range(D)] for t in range(B)])


class Cache:
    """Token-ordered numbers of every block: codes [n_blocks][kv_heads][B][D] and exponents [n_blocks][kv_heads]."""

    def __init__(self, n_blocks, B, kv, D):
        self.n_blocks, self.B, self.kv, self.D = n_blocks, B, kv, D
        self.codes = [np.zeros((n_blocks, kv, B, D), np.uint8) for _ in range(2)]
        self.exps = [np.full((n_blocks, kv), EXP_MIN, np.int64) for _ in range(2)]

    def append(self, rows, slots):
        """rows: [keys, values], each [T][kv][D] float64."""
        t = 0
        while t < len(slots):
            s = int(slots[t])
            if s < 0 or s // self.B >= self.n_blocks:
                t += 1
                continue
            b, off, m = s // self.B, s % self.B, 1
            while t + m < len(slots) and slots[t + m] == s + m and off + m < self.B:
                m += 1
            for w in range(2):
                for h in range(self.kv):
                    x = rows[w][t:t + m, h]
                    fin = np.abs(x[np.isfinite(x)])
                    e = exponent(fin.max() if fin.size else 0.0)
                    if off > 0:
                        old = self.exps[w][b, h]
                        e = max(e, old)
                        if e > old:
                            self.codes[w][b, h, :off] = encode(np.ldexp(VALUES[self.codes[w][b, h, :off]], old - e))
                    self.exps[w][b, h] = e
                    self.codes[w][b, h, off:off + m] = encode(np.ldexp(x, -int(e)))
            t += m

    def tokens(self, w, slots):
        """[len(slots)][kv][D]; zeros for slots outside."""
        slots = np.asarray(slots, np.int64)
        there = (slots >= 0) & (slots // self.B < self.n_blocks)
        b, t = np.where(there, slots // self.B, 0), np.where(there, slots % self.B, 0)
        out = np.ldexp(VALUES[self.codes[w][b, :, t]], self.exps[w][b][:, :, None])
        out[~there] = 0.0
        return out

    def pages(self, w):
        """The bytes as the library lays them out, and the scale bytes."""
        at = places(self.B, self.D, w == 1)
        out = np.empty((self.n_blocks, self.kv, self.B * self.D), np.uint8)
        out[:, :, at.reshape(-1)] = self.codes[w].reshape(self.n_blocks, self.kv, -1)
        return out, (self.exps[w] + 127).astype(np.uint8)


def plan(cached, fresh, free, table, B, max_tokens):
    """table is changed in place; returns (lengths, starts, slots, positions, taken)."""
    n, width = table.shape
    slots, positions = np.full(max_tokens, -1, np.int64), np.full(max_tokens, -1, np.int64)
    lengths, starts, t, taken = [], [0], 0, 0
    for r in range(n):
        c, f = max(int(cached[r]), 0), max(int(fresh[r]), 0)
        had, has = min(-(-c // B), width), min(-(-(c + f) // B), width)
        for b in range(had, has):
            entry = int(free[taken]) if taken < len(free) else -1
            taken += 1
            first = b * B                        # written by the row of its first token, if that row is held
            if t + first - c < max_tokens:
                table[r, b] = entry
        for i in range(f):
            p = c + i
            if t < max_tokens:
                positions[t] = p
                if p // B < width:
                    # (a block that lies past max_tokens' rows was not entered, and none of its rows is held)
                    e = int(table[r, p // B])
                    slots[t] = e * B + p % B if e >= 0 else -1
            t += 1
        lengths.append(c + f)
        starts.append(t)
    return np.array(lengths), np.array(starts), slots, positions, taken


def attention(cache: Cache, q, table, lengths, starts, group, scale, window=0):
    """q [T][heads][D] float64 -> out [T][heads][D]; rows past starts[-1] are NaN."""
    T, heads, D = q.shape
    out = np.full((T, heads, D), np.nan)
    for r in range(len(lengths)):
        f, L = int(starts[r + 1] - starts[r]), int(lengths[r])
        slots = []
        for j in range(L):
            e = int(table[r, j // cache.B]) if j // cache.B < table.shape[1] else -1
            slots.append(e * cache.B + j % cache.B if 0 <= e < cache.n_blocks else -1)
        slots = np.array(slots, np.int64)
        there = slots >= 0
        K, V = (cache.tokens(w, slots) for w in range(2))
        j = np.arange(L)
        for i in range(f):
            p = L - f + i
            see = (j <= p) & there
            if window:
                see &= j > p - window
            t = int(starts[r]) + i
            if not see.any():
                out[t] = 0.0
                continue
            with np.errstate(all="ignore"):
                s = np.einsum("hd,jhd->hj", q[t], np.repeat(K[see], group, axis=1)) * scale
                s = np.exp(s - s.max(axis=1, keepdims=True))
                s /= s.sum(axis=1, keepdims=True)
                out[t] = np.einsum("hj,jhd->hd", s, np.repeat(V[see], group, axis=1))
    return out
