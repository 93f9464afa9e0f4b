"""Absorbed attention of parts of hundreds of steps, every step seen: a row's query points at one token, which rules its softmax, and the rows'
tokens go through all steps.  A step left out, or a block read in the place of another, is then an error of the size of a latent; the first
test shows on the CPU that the bound refuses each such mistake."""
import numpy as np
import pytest
import torch

from oracle import latent_oracle as L
from kv_util import act_round
from latent_util import Absorbed, softmax_reference

KEYS, B, STEP = 20001, 128, 64
# Scores of the token pointed at and of others differ by |k|^2 - k . k', at least 150 of about 350 for latents of 256 (five deviations
# of either): times 0.15 that is e^22, so that twenty thousand others together weigh 1e-5 of it.
POINTED = 0.15


class Pointed(Absorbed):
    """`n` requests of 17000 to 20001 tokens over the same blocks, one new token each."""

    def __init__(self, act, heads, latent, n):
        rng = np.random.default_rng(19)
        super().__init__(rng, [(KEYS - 1, 1)], heads, latent, 32, B, act, spread=0)
        self.slots = L.slots_of(self.table, 0, KEYS, B, self.cache.n_blocks)
        self.lat = self.cache.latents(self.slots)
        self.k = np.concatenate([self.lat, self.cache.key_parts(self.slots)], 1)
        self.exp = self.cache.exps[self.slots].astype(np.float64)
        self.fresh, self.lengths = [1] * n, [int(v) for v in rng.integers(17000, KEYS + 1, n)]
        self.lengths[0] = KEYS
        self.starts, self.T, self.table = np.arange(n + 1), n + 1, np.repeat(self.table, n, 0)
        # row i of all (request, head) points at step 97 i, which goes through all 313, or as far into its request as that has steps
        steps = np.repeat([-(-v // STEP) for v in self.lengths], heads)
        first = np.arange(n * heads) * 97 % -(-KEYS // STEP) % steps * STEP
        last = np.minimum(first + STEP, np.repeat(self.lengths, heads))
        self.at = (first + rng.integers(0, 1 << 30, n * heads) % (last - first)).reshape(n, heads)
        self.q = np.zeros((self.T, heads, latent + 32))
        self.q[:n] = act_round(self.k[self.at] * (POINTED / self.scale), act)

    def reference(self, device="cuda"):
        k, lat, e = (torch.from_numpy(x).to(device) for x in (self.k, self.lat, self.exp))
        out, bound = np.zeros((len(self.fresh), self.heads, self.latent)), np.zeros((len(self.fresh), self.heads, self.latent))
        for r, n in enumerate(self.lengths):
            see = torch.ones(self.heads, n, dtype=torch.bool, device=device)
            o, b = softmax_reference(torch.from_numpy(self.q[r]).to(device), k[:n], lat[:n].contiguous(), see, self.scale, self.act, self.latent + self.rope, e[:n])
            out[r], bound[r] = o.cpu().numpy(), b.cpu().numpy()
        return out, bound


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("heads,latent", [(40, 256), (8, 512)])
def test_the_bound_refuses_wrong_steps_and_blocks(act, heads, latent):
    b = Pointed(act, heads, latent, 300)
    # every step, and each quarter of steps, has several rows that point at it
    assert (np.bincount(b.at.reshape(-1) // STEP)[:17000 // STEP] >= 5).all() and len(np.unique(b.at % STEP // 16)) == 4
    assert (b.at < np.array(b.lengths)[:, None]).all()
    one = Pointed(act, heads, latent, 1)
    steps = -(-KEYS // STEP)
    at = np.minimum(np.arange(steps) * STEP + 11, KEYS - 1)
    one.heads, one.q = steps, act_round(one.k[at] * (POINTED / one.scale), act)[None]
    want, bound = (x[0] for x in one.reference("cpu"))
    assert (np.abs(want - one.lat[at]) < 0.02).all()
    s = one.q[0] @ one.k.T * one.scale
    w = np.exp(s - s.max(1, keepdims=True))
    blocks = -(-KEYS // B)
    for t in range(steps):
        here = slice(STEP * t, min(STEP * (t + 1), KEYS))
        gone = w[t].copy()
        gone[here] = 0.0
        # a block read in the place of the row's: its neighbour, as many tokens as the row's has
        blk = at[t] // B
        other = blk - 1 if blk + 1 >= blocks else blk + 1
        m = min(B, KEYS - B * blk, KEYS - B * other)
        moved = w[t].copy()
        moved[B * blk:B * blk + B] = 0.0
        moved[B * other:B * other + m] *= 2.0
        for name, x in (("left out", gone), ("another block", moved)):
            got = x @ one.lat / x.sum()
            assert (np.abs(got - want[t]) > bound[t]).any(), (name, t)
            assert (np.abs(got - want[t]) > 3 * bound[t]).mean() > 0.5, (name, t)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("heads,latent", [(40, 256), (8, 512)])
def test_absorbed_sees_every_step_of_long_parts(act, heads, latent):
    b = Pointed(act, heads, latent, 300)                           # more units than the machine holds: parts of 130 to 313 steps
    b.device().run().check()
