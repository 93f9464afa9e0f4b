"""Expanded attention, binary16: a first token that rules every softmax and adds nothing, before a long context.  As for absorbed attention
(test_latent_sinks.py derives the bound), but for the sum of the weights: it is that of the numbers that are multiplied."""
import math

import numpy as np
import pytest

from kv_util import act_round
from latent_util import Expanded
from test_latent_sinks import BITS, HELD, KEYS, bound


class Sink(Expanded):
    def __init__(self, n_requests, heads=len(BITS)):
        rng = np.random.default_rng(29)
        super().__init__(rng, [(KEYS - 1, 1)], heads, 64, 32, "f16")
        self.k[:KEYS], self.kr[:KEYS], self.v[:KEYS] = 0.0, 0.0, act_round(rng.uniform(1.0, 1.75, (KEYS, heads, 64)), "f16")
        self.v[0] = 0.0
        self.kr[1:KEYS, 1], self.kr[0, 0] = act_round(rng.uniform(-0.5, 0.5, KEYS - 1), "f16"), 1.0
        # all requests read the same keys
        self.fresh, self.lengths, self.starts, self.T = [1] * n_requests, [KEYS] * n_requests, np.arange(n_requests + 1), n_requests + 1
        self.key_starts = np.zeros(n_requests, int)
        q = np.zeros((heads, 96))
        q[:, 64], q[:, 65] = BITS[:heads] * math.log(2.0) / self.scale, math.log(2.0) / self.scale
        self.q = np.repeat(act_round(q, "f16")[None], self.T, 0)
        s = (self.kr[:KEYS] @ self.q[0, :, 64:].T * self.scale / math.log(2.0)).T     # base 2
        self.w = np.exp2(s - s.max(1, keepdims=True))
        self.want = self.sums(self.w) / self.w.sum(1)[:, None]

    def sums(self, w):
        return np.stack([w[h] @ self.v[:KEYS, h] for h in range(self.heads)])

    def error(self, got):
        return np.sqrt(((got - self.want) ** 2).mean(1) / (self.want ** 2).mean(1))


def test_weights_held_lower_are_refused():
    b = Sink(1)
    for held in (0, HELD):
        p = act_round(b.w * 2.0 ** held, "f16") * 2.0 ** -held
        right = b.error(act_round(b.sums(p) / p.sum(1)[:, None], "f16")) <= bound(KEYS)
        assert right.all() if held else not right[BITS >= 25].any(), held


@pytest.mark.gpu
def test_expanded_after_a_token_that_rules_and_adds_nothing():
    b = Sink(43)                                                    # 516 units: as many as shares, so that none is cut
    out = b.device().run().output()
    assert (out == out[0]).all()
    error = b.error(out[0])
    print("error:", " ".join(f"{x:.1e}" for x in error))
    assert (error <= bound(KEYS)).all(), (error / bound(KEYS)).tolist()
