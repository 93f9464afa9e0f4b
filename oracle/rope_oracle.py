"""Slow CPU oracle of rotary positions: frequencies of every scaling, rotation of rows.  float64, one pair at a time; written
from the definitions in include/glowq.h and sharing nothing with the kernels."""
from __future__ import annotations

import math

import numpy as np


def frequencies(r, base, scaling="plain", factor=1.0, low=0.0, high=0.0, length=0):
    """(f_i for i < r / 2, magnitude)"""
    if scaling == "rebased":
        base = base * factor ** (r / (r - 2))
    out = []
    for i in range(r // 2):
        f = base ** (-2.0 * i / r)
        if scaling == "stretched":
            f = f / factor
        elif scaling == "bands":
            n = length * f / (2 * math.pi)
            fast = min(max((n - low) / (high - low), 0.0), 1.0)
            f = fast * f + (1 - fast) * f / factor
        elif scaling == "ramp":
            # the pair that makes n turns over the trained length: length base^(-2 i / r) / 2 pi = n
            pair = lambda n: r / 2 * math.log(length / (2 * math.pi * n), base)
            first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), r - 1)
            slow = min(max((i - first) / max(last - first, 0.001), 0.0), 1.0)
            f = slow * f / factor + (1 - slow) * f
        out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1 if scaling == "ramp" else 1.0


def angles(turns, positions):
    """Angles [positions][pairs], each within a turn, of frequencies as 64-bit fractions of one."""
    return np.array([[int(p) * int(t) % (1 << 64) / 2.0 ** 64 * 2 * math.pi for t in turns] for p in positions]).reshape(len(positions), len(turns))


def pairs_of(r, layout):
    """dims (a, b) of every pair"""
    return [(i, i + r // 2) if layout == "halves" else (2 * i, 2 * i + 1) for i in range(r // 2)]


def rotate(x, turns, positions, layout, magnitude=1.0):
    """x [T][heads][dims] float64; rows at negative positions as they are."""
    y, r = np.array(x, np.float64), 2 * len(turns)
    at = angles(turns, positions)
    for t, p in enumerate(positions):
        if p < 0:
            continue
        for i, (a, b) in enumerate(pairs_of(r, layout)):
            c, s = math.cos(at[t, i]) * magnitude, math.sin(at[t, i]) * magnitude
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, a] * s + x[t, :, b] * c
    return y


def reach(x, r, layout, magnitude=1.0):
    """|a| + |b| of the pair that each number lies in, times the magnitude: what an error of sine and cosine is multiplied with."""
    out = np.zeros_like(x)
    for a, b in pairs_of(r, layout):
        out[..., a] = out[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(magnitude)
    return out
