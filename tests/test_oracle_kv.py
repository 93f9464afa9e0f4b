"""Pins of the serving operators' oracle: codes against the library's cast, pages as a permutation, exponents, plans by
hand, attention in special cases."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as K


def test_codes_are_the_library_cast():
    rng = np.random.default_rng(1)
    x = np.concatenate([K.MAGNITUDES, (K.MAGNITUDES[:-1] + K.MAGNITUDES[1:]) / 2, rng.uniform(0, 448, 4000),
                        2.0 ** rng.uniform(-12, 8, 4000)]).astype(np.float32).astype(np.float64)
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(K.encode(x), want)
    assert np.array_equal(K.VALUES[:127], torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    assert (K.encode(np.array([np.inf, -np.inf, np.nan])) == K.NAN_CODE).all()


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (224.0, -1), (1.75, -8), (1.7500001, -7), (0.0, K.EXP_MIN), (1e-30, K.EXP_MIN),
                                   (65504.0, 8), (2.9e38, 119), (3.0e38, 120)])
def test_exponents(top, e):
    assert K.exponent(top) == e
    assert top <= math.ldexp(448.0, e) and (e == K.EXP_MIN or top > math.ldexp(448.0, e - 1))


@pytest.mark.parametrize("B,D", [(16, 64), (32, 128), (128, 64)])
def test_pages_hold_every_byte_once(B, D):
    for values in (False, True):
        assert np.array_equal(np.sort(K.places(B, D, values).reshape(-1)), np.arange(B * D))
    assert K.key_byte(17, 70, 128) == 3 * 1024 + 1 * 16 + 6 and K.value_byte(17, 70, 128) == 3 * 1024 + 6 * 16 + 1
    assert K.key_byte(5, 35, 64) == 2 * 256 + 5 * 16 + 3 and K.value_byte(5, 35, 64) == 1 * 256 + 3 * 16 + 2 * 4 + 1


def test_appending_in_parts_gives_the_same_numbers_as_at_once():
    rng = np.random.default_rng(2)
    x = [rng.standard_normal((40, 2, 64)) * 2.0 ** rng.integers(-2, 3, (40, 1, 1)) for _ in range(2)]
    slots = np.arange(32, 72)
    whole, parts = K.Cache(5, 32, 2, 64), K.Cache(5, 32, 2, 64)
    whole.append(x, slots)
    for t in range(0, 40, 3):
        parts.append([v[t:t + 3] for v in x], slots[t:t + 3])
    for w in range(2):
        assert np.array_equal(whole.exps[w][1:3], parts.exps[w][1:3])
        a, b = whole.tokens(w, slots), parts.tokens(w, slots)
        step = np.ldexp(2.0 ** -9, whole.exps[w][slots // 32])[..., None]
        assert (np.abs(a - b) <= step).all()                     # subnormal codes may round twice
        assert (np.abs(a - x[w]) <= np.maximum(np.abs(x[w]) * 2.0 ** -4, step / 2)).all()


def test_a_plan_by_hand():
    table = np.full((3, 4), -1)
    table[0, 0], table[2, :2] = 7, (3, 9)
    lengths, starts, slots, positions, taken = K.plan([15, 0, 30], [3, 0, 1], [4, 5], table, 16, 6)
    assert lengths.tolist() == [18, 0, 31] and starts.tolist() == [0, 3, 3, 4] and taken == 1
    assert positions.tolist() == [15, 16, 17, 30, -1, -1]
    assert slots.tolist() == [7 * 16 + 15, 4 * 16, 4 * 16 + 1, 9 * 16 + 14, -1, -1]
    assert table.tolist() == [[7, 4, -1, -1], [-1] * 4, [3, 9, -1, -1]]
    short = np.full((1, 4), -1)
    _, _, slots, _, taken = K.plan([0], [40], [2], short, 16, 40)
    assert taken == 3 and slots[:16].tolist() == list(range(32, 48)) and (slots[16:] == -1).all() and short.tolist() == [[2, -1, -1, -1]]


def test_attention_in_special_cases():
    rng = np.random.default_rng(3)
    c = K.Cache(4, 16, 1, 64)
    x = [rng.standard_normal((40, 1, 64)) for _ in range(2)]
    table = np.array([[2, 0, 3]])
    slots = table[0][np.arange(40) // 16] * 16 + np.arange(40) % 16
    c.append(x, slots)
    V = c.tokens(1, slots)[:, 0]
    q = np.zeros((2, 2, 64))
    out = K.attention(c, q, table, [40], [0, 2], 2, 0.125)
    assert np.allclose(out[1], V.mean(0)) and np.allclose(out[0], V[:39].mean(0))               # equal scores: the mean
    assert np.allclose(K.attention(c, q, table, [40], [0, 2], 2, 0.125, window=1)[1], V[39])    # one key: its value
    q[:, 0] = 100.0 * c.tokens(0, slots)[5, 0]
    assert np.allclose(K.attention(c, q, table, [40], [0, 2], 2, 1.0)[:, 0], V[5])              # one key far ahead
    assert (K.attention(c, q, table, [1], [0, 2], 2, 1.0)[0] == 0).all()                        # p < 0: nothing seen
