"""The oracles of rotary positions and latent attention against what defines them: on the CPU."""
import math
from fractions import Fraction

import numpy as np
import pytest

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from oracle import latent_oracle as L
from oracle import rope_oracle as R

SCALINGS = {"plain": (10000.0, 1.0, 0.0, 0.0, 0), "stretched": (10000.0, 4.0, 0.0, 0.0, 0), "rebased": (10000.0, 8.0, 0.0, 0.0, 0),
            "bands": (500000.0, 8.0, 1.0, 4.0, 8192), "ramp": (10000.0, 40.0, 1.0, 32.0, 4096)}
KINDS = {"plain": G.GLOWQ_ROPE_PLAIN, "stretched": G.GLOWQ_ROPE_STRETCHED, "rebased": G.GLOWQ_ROPE_REBASED, "bands": G.GLOWQ_ROPE_BANDS,
         "ramp": G.GLOWQ_ROPE_RAMP}


def spec(r, scaling):
    base, factor, low, high, length = SCALINGS[scaling]
    return G.make_rope_spec(rotary_dim=r, scaling=KINDS[scaling], base=base, factor=factor, low=low, high=high, trained_length=length)


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("r", [16, 64, 128, 256])
def test_turns_are_the_frequencies(r, scaling):
    base, factor, low, high, length = SCALINGS[scaling]
    f, magnitude = R.frequencies(r, base, scaling, factor, low, high, length)
    turns, m = G.glowq_rope_turns(spec(r, scaling))
    assert len(turns) == r // 2 and abs(m - magnitude) <= 2.0 ** -24 * magnitude
    # the oracle's powers and logarithms are good to a few 2^-53 times their exponent (14 at most); a turn is kept to half of 2^-64
    assert np.allclose(np.array([t / 2.0 ** 64 for t in turns]) * 2 * math.pi, f, rtol=2.0 ** -46, atol=2 * math.pi * 2.0 ** -65)


def test_scalings_move_what_they_should():
    r = 128
    plain = R.frequencies(r, 10000.0)[0]
    rebased = R.frequencies(r, 10000.0, "rebased", 8.0)[0]
    assert plain[0] == rebased[0] == 1.0 and abs(rebased[-1] * 8 / plain[-1] - 1) < 1e-12
    base = R.frequencies(r, 500000.0)[0]
    bands = R.frequencies(r, 500000.0, "bands", 8.0, 1.0, 4.0, 8192)[0]
    turns = 8192 * base / (2 * math.pi)
    assert np.allclose(bands[turns >= 4], base[turns >= 4]) and np.allclose(bands[turns <= 1], base[turns <= 1] / 8)
    assert np.all((bands <= base * (1 + 1e-12)) & (bands >= base / 8 * (1 - 1e-12)))
    ramp, m = R.frequencies(r, 10000.0, "ramp", 40.0, 1.0, 32.0, 4096)
    turns = 4096 * plain / (2 * math.pi)
    assert np.allclose(ramp[turns >= 32 * 1.2], plain[turns >= 32 * 1.2]) and np.allclose(ramp[turns <= 1 / 1.2], plain[turns <= 1 / 1.2] / 40)
    assert m == 0.1 * math.log(40.0) + 1


def test_angles_are_exact_at_any_position():
    turns = [12345678901234567890 // 7, 1 << 61, 3]
    for p in (0, 1, 131071, (1 << 31) - 1):
        for t, a in zip(turns, R.angles(turns, [p])[0]):
            want = Fraction(p * t, 1 << 64) % 1
            assert abs(a - float(want) * 2 * math.pi) < 1e-14


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_rotation_keeps_lengths_and_differences_of_positions(layout):
    rng = np.random.default_rng(1)
    turns, _ = G.glowq_rope_turns(spec(32, "plain"))
    q, k = rng.standard_normal((2, 1, 1, 48))
    dot = lambda p, j: float(R.rotate(q, turns, [p], layout).ravel() @ R.rotate(k, turns, [j], layout).ravel())
    assert abs(dot(7, 3) - dot(107, 103)) < 1e-12 and abs(dot(7, 3) - dot(8, 3)) > 1e-3
    y = R.rotate(q, turns, [1000], layout)
    assert np.array_equal(y[..., 32:], q[..., 32:]) and abs(np.linalg.norm(y) - np.linalg.norm(q)) < 1e-12
    assert np.array_equal(R.rotate(q, turns, [-1], layout), q) and np.array_equal(R.rotate(q, turns, [0], layout), q)


@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_a_token_is_on_the_finest_grid_that_holds_it(act):
    rng = np.random.default_rng(2)
    for top in (0.0, 1e-5, 0.3, 448.0, 449.0, 60000.0, 65504.0):
        c = rng.uniform(-1, 1, 256) * top
        c[3] = top
        e = L.exponent(c, act)
        assert top <= math.ldexp(448.0, e) and (e in (-15, -64) or top > math.ldexp(448.0, e - 1))
        cache = L.LatentCache(1, 16, 256, 32, act)
        cache.append(c[None], np.zeros((1, 32)), [5])
        x = cache.latents([5])[0]
        most = 61440.0 if act == "f16" else np.inf
        assert np.all(np.abs(x - c) <= np.maximum(np.abs(c) * 2.0 ** -4, math.ldexp(1.0, e - 10))) and np.abs(x).max() <= most
    c[7], c[9] = np.inf, np.nan
    cache.append(c[None], np.zeros((1, 32)), [6])
    assert np.array_equal(np.isnan(cache.latents([6])[0]), ~np.isfinite(c)) and not cache.latents([16]).any()


def test_both_forms_are_one_attention():
    rng = np.random.default_rng(3)
    heads, N, latent, rope = 3, 8, 256, 32
    cache = L.LatentCache(4, 16, latent, rope, "bf16")
    cache.codes[:] = K.encode(np.clip(rng.standard_normal(cache.codes.shape) * 72, -448, 448))
    cache.exps[:], cache.ropes[:] = -6, rng.standard_normal(cache.ropes.shape)
    table, lengths, starts = np.array([[2, 0], [3, -1]]), [21, 9], [0, 3, 5]
    U, V, q = rng.standard_normal((heads, N, latent)) / 16, rng.standard_normal((heads, N, latent)) / 16, rng.standard_normal((5, heads, N + rope))
    qa = np.concatenate([np.einsum("thn,hnl->thl", q[..., :N], U), q[..., N:]], -1)
    a = np.einsum("thl,hnl->thn", L.absorbed(cache, qa, table, lengths, starts, 0.2), V)
    slots = np.concatenate([L.slots_of(table, r, n, 16, 4) for r, n in enumerate(lengths)])
    lat = cache.latents(slots)
    e = L.expanded(q, np.einsum("jl,hnl->jhn", lat, U), cache.key_parts(slots), np.einsum("jl,hnl->jhn", lat, V), starts, [0, 21], lengths, 0.2)
    assert np.allclose(a, e, rtol=1e-10, atol=1e-12)
