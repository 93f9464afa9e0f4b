"""Absorbed attention, binary16: a first token that rules every softmax and adds (nearly) nothing, before a long context whose tokens weigh 2^-16
to 2^-27 of it each.  What those add up to is nearly all of the output; the error is looked at relative to that.

The weights are multiplied as binary16 numbers, of which the smallest is 2^-24: with the row's largest held at 2^7 to 2^15, a weight d bits
below is at least U = 2^(31 - d) such steps.  Errors, relative to the output's norm:
  - two roundings by 2^-11, of the output and of the ruling weight;
  - the others' roundings, half a step each, over tokens whose weights are spread evenly over a factor of two (in bits: U / sqrt 2 to U sqrt 2):
    what does not average out is the error of a step's two cut-off ends, an eighth of a step each at a density of 1 / (ln 2 U / sqrt 2),
    and six deviations of n independent ones;
  - scores in fp32: 2^-18 counts sixty-four last places of them.
"""
import math

import numpy as np
import pytest

from oracle import latent_oracle as L
from kv_util import act_round
from latent_util import Absorbed

KEYS, HELD = 100001, 7
BITS = np.arange(16, 28)               # of the ruling token above the others, head by head


def bound(n):
    u = 2.0 ** (24 + HELD - BITS)
    low = u / math.sqrt(2.0)
    return 2 * 2.0 ** -11 + 0.25 / (math.log(2.0) * low * u) + 6 * 0.5 / low / np.sqrt(3.0 * n) + 2.0 ** -18


class Sink(Absorbed):
    def __init__(self, n_requests):
        rng = np.random.default_rng(23)
        super().__init__(rng, [(KEYS - 1, 1)], len(BITS), 256, 32, 128, "f16", spare=0)
        slots = L.slots_of(self.table, 0, KEYS, 128, self.cache.n_blocks)
        c, r = rng.uniform(1.0, 1.75, (KEYS, 256)), np.zeros((KEYS, 32))
        c[:, 0] = 1.75                                              # (so that all have the same scale)
        c[0, 1:] = 0.0
        r[1:, 1], r[0, 0] = rng.uniform(-0.5, 0.5, KEYS - 1), 1.0
        self.cache.append(act_round(c, "f16"), act_round(r, "f16"), slots)
        assert (self.cache.exps[slots] == -8).all()
        self.fresh, self.lengths, self.starts, self.T = [1] * n_requests, [KEYS] * n_requests, np.arange(n_requests + 1), n_requests + 1
        self.table = np.repeat(self.table, n_requests, 0)
        q = np.zeros((len(BITS), 288))
        q[:, 256], q[:, 257] = BITS * math.log(2.0) / self.scale, math.log(2.0) / self.scale
        self.q = np.repeat(act_round(q, "f16")[None], self.T, 0)
        self.lat = self.cache.latents(slots)
        s = (self.cache.key_parts(slots) @ self.q[0, :, 256:].T * self.scale / math.log(2.0)).T     # base 2
        self.w = np.exp2(s - s.max(1, keepdims=True))
        self.want = self.w @ self.lat / self.w.sum(1)[:, None]

    def error(self, got):
        """Of what the others add up to, per head."""
        off, size = got[:, 1:] - self.want[:, 1:], self.want[:, 1:]
        return np.sqrt((off ** 2).mean(1) / (size ** 2).mean(1))


def test_weights_held_lower_are_refused():
    b = Sink(1)
    for held in (0, HELD):
        # the formula with weights as binary16 numbers, their sum of 11 bits each
        p = act_round(b.w * 2.0 ** held, "f16") * 2.0 ** -held
        m, e = np.frexp(b.w)
        got = act_round(p @ b.lat / np.ldexp(np.round(m * 2048) / 2048, e).sum(1)[:, None], "f16")
        right = b.error(got) <= bound(KEYS)
        assert right.all() if held else not right[BITS >= 24].any(), (held, b.error(got) / bound(KEYS))


@pytest.mark.gpu
def test_absorbed_after_a_token_that_rules_and_adds_nothing():
    b = Sink(300)                                                   # more units than the machine holds: none is cut
    out = b.device().run().output()
    assert (out == out[0]).all()
    error = b.error(out[0])
    print("error:", " ".join(f"{x:.1e}" for x in error))
    assert (error <= bound(KEYS)).all(), (error / bound(KEYS)).tolist()
