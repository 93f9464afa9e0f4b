"""Calls that the header allows at the edge of what the positions and expanded attention take: numbers beside the rotated ones bit by bit, requests
beyond the caller's bounds, requests whose keys would lie behind the last row."""
import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from gpu_util import ACT_CODE, TORCH_ACT, stream
from kv_util import i32
from latent_util import Expanded, Rope, softmax_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_numbers_behind_the_rotated_ones_keep_their_bits(act, layout):
    rng, T, h, d, r = np.random.default_rng(1), 37, 3, 96, 32
    bits = torch.int32 if act == "f32" else torch.int16
    x = torch.randn(T, h, d, device="cuda").to(TORCH_ACT[act])
    # every kind of number: subnormal ones, zeros of either sign, infinities
    odd = torch.tensor([1, 3, -(1 << (31 if act == "f32" else 15)), 0], dtype=torch.int64).to(bits).cuda()
    x.view(bits)[:, :, r:r + 4] = odd
    x[:, :, r + 4], x[:, :, r + 5] = float("inf"), -float("inf")
    x[:, :, d - 1] = float("nan")
    y, positions = torch.zeros_like(x), i32(rng.integers(0, 1 << 20, T))
    rows = G.make_rope_rows(x=x.data_ptr(), y=y.data_ptr(), heads=h, ldx=h * d, lhx=d, ldy=h * d, lhy=d)
    G.glowq_rotate(Rope(r, layout).desc, [rows], d, ACT_CODE[act], positions.data_ptr(), T, stream())
    torch.cuda.synchronize()
    assert torch.equal(y.view(bits)[:, :, r:d - 1], x.view(bits)[:, :, r:d - 1]) and torch.isnan(y[:, :, d - 1]).all()


@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_expanded_beyond_the_callers_bounds(act):
    b = Expanded(np.random.default_rng(2), [(100, 5), (20, 2)], 3, 64, 32, act)
    out = b.device(max_fresh=2, max_length=64).run().output()
    assert np.isnan(out[2:5]).all()                                # rows past max_fresh stay unwritten
    # keys past max_length are left out, rows keep their positions
    for r, at, n in ((0, 0, 64), (1, 5, 22)):
        k0 = int(b.key_starts[r])
        see = torch.arange(n)[None] <= torch.arange(b.lengths[r] - b.fresh[r], b.lengths[r] - b.fresh[r] + 2)[:, None]
        for h in range(3):
            k = torch.from_numpy(np.concatenate([b.k[k0:k0 + n, h], b.kr[k0:k0 + n]], 1))
            want, bound = softmax_reference(torch.from_numpy(b.q[at:at + 2, h]), k, torch.from_numpy(b.v[k0:k0 + n, h]).contiguous(), see, b.scale, act, 96)
            assert (np.abs(out[at:at + 2, h] - want.numpy()) <= bound.numpy()).all()


def test_expanded_keys_that_are_not_there():
    # the second request's keys would begin behind the last row, the third's end behind it
    b = Expanded(np.random.default_rng(3), [(60, 4), (30, 3), (10, 150)], 2, 128, 64, "bf16", extra_keys=0)
    b.key_starts[1], b.key_starts[2] = b.keys, b.keys - 100
    for x in (b.k, b.v, b.kr):
        x[np.isnan(x)] = 0.0
    out = b.device().run().output()
    assert not out[4:7].any()
    for i in (0, 80, 89, 90, 149):                                 # of the third: it has 100 keys
        n = min(10 + i + 1, 100)
        k0 = b.keys - 100
        for h in range(2):
            k = torch.from_numpy(np.concatenate([b.k[k0:k0 + n, h], b.kr[k0:k0 + n]], 1))
            want, bound = softmax_reference(torch.from_numpy(b.q[7 + i:8 + i, h]), k, torch.from_numpy(b.v[k0:k0 + n, h]).contiguous(), torch.ones(1, n, dtype=torch.bool),
                                            b.scale, "bf16", 192)
            assert (np.abs(out[7 + i, h] - want.numpy()) <= bound.numpy()).all()
