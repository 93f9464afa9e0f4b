"""Slow CPU oracle of the latent cache and of latent attention in both forms.  numpy, float64; written from the definitions in
include/glowq.h and sharing nothing with the kernels."""
from __future__ import annotations

import math

import numpy as np

from oracle import kv_oracle as K

# the largest code value of the type: the code behind 240 stands for 256, 2^16 and 2^128
MOST = {"f16": 61440.0, "bf16": 240 * 2.0 ** 120}


def exponent(c, act):
    """Of one token's latent: the smallest e with max |c| <= 448 * 2^e over its finite numbers, at least -64 (f16: -15)."""
    fin = np.abs(c[np.isfinite(c)])
    return max(K.exponent(fin.max() if fin.size else 0.0), -15 if act == "f16" else -64)


class LatentCache:
    """codes [slots][latent], exponents [slots], ropes [slots][rope] (float64 of the cache's type)"""

    def __init__(self, n_blocks, B, latent, rope, act):
        self.n_blocks, self.B, self.latent, self.rope, self.act = n_blocks, B, latent, rope, act
        self.codes = np.zeros((n_blocks * B, latent), np.uint8)
        self.exps = np.full(n_blocks * B, -15, np.int64)
        self.ropes = np.zeros((n_blocks * B, rope))

    def append(self, c, r, slots):
        """Rows c [T][latent], r [T][rope] (already rotated)."""
        for t, s in enumerate(slots):
            if 0 <= s < len(self.exps):
                e = exponent(c[t], self.act)
                x = np.ldexp(c[t], -e)
                x = np.where(np.isfinite(x), np.clip(x, np.ldexp(-MOST[self.act], -e), np.ldexp(MOST[self.act], -e)), x)
                self.codes[s], self.exps[s], self.ropes[s] = K.encode(x), e, r[t]

    def latents(self, slots):
        """[len(slots)][latent]; zeros for slots outside."""
        slots = np.asarray(slots, np.int64)
        there = (slots >= 0) & (slots < len(self.exps))
        at = np.where(there, slots, 0)
        out = np.ldexp(K.VALUES[self.codes[at]], self.exps[at][:, None])
        out[~there] = 0.0
        return out

    def key_parts(self, slots):
        slots = np.asarray(slots, np.int64)
        there = (slots >= 0) & (slots < len(self.exps))
        return np.where(there[:, None], self.ropes[np.where(there, slots, 0)], 0.0)


def slots_of(table, r, length, B, n_blocks):
    """Slots of a request's tokens; -1 where its block is outside the cache."""
    out = []
    for j in range(max(length, 0)):
        e = int(table[r, j // B]) if j // B < table.shape[1] else -1
        out.append(e * B + j % B if 0 <= e < n_blocks else -1)
    return np.array(out, np.int64)


def _attend(q, k, v, see, scale):
    """One row and head."""
    if not see.any():
        return np.zeros(v.shape[1])
    with np.errstate(all="ignore"):
        s = k[see] @ q * scale
        s = np.exp(s - s.max())
        return s @ v[see] / s.sum()


def absorbed(cache, q, table, lengths, starts, scale):
    """q [T][heads][latent + rope] -> [T][heads][latent]; rows past starts[-1] are NaN."""
    T, heads, _ = q.shape
    out = np.full((T, heads, cache.latent), np.nan)
    for r, L in enumerate(lengths):
        slots = slots_of(table, r, int(L), cache.B, cache.n_blocks)
        lat = cache.latents(slots)
        k = np.concatenate([lat, cache.key_parts(slots)], 1)
        f = int(starts[r + 1] - starts[r])
        for i in range(f):
            see = (slots >= 0) & (np.arange(len(slots)) <= int(L) - f + i)
            for h in range(heads):
                out[starts[r] + i, h] = _attend(q[starts[r] + i, h], k, lat, see, scale)
    return out


def expanded(q, k, kr, v, starts, key_starts, lengths, scale):
    """q [T][heads][nope + rope], k [keys][heads][nope], kr [keys][rope], v [keys][heads][dims]."""
    T, heads, _ = q.shape
    out = np.full((T, heads, v.shape[2]), np.nan)
    for r, L in enumerate(lengths):
        f, L = int(starts[r + 1] - starts[r]), max(int(L), 0)
        at = slice(int(key_starts[r]), int(key_starts[r]) + L)
        for i in range(f):
            see = np.arange(L) <= int(lengths[r]) - f + i
            for h in range(heads):
                keys = np.concatenate([k[at, h], kr[at]], 1)
                out[starts[r] + i, h] = _attend(q[starts[r] + i, h], keys, v[at, h], see, scale)
    return out
