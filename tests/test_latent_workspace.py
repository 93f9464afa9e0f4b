"""Workspace of absorbed attention: a partial result for every part that leaves one, not for every tile of rows."""
import random

import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from latent_util import Absorbed

PLACES, LEAST, STEP = 256, 2, 64
MOST = 640                             # partial results: 2.5 for every workgroup that the machine holds


def cut(units):
    """(parts, parts that leave partial results) of units with so many steps each, as the header of the cut states it: parts of an equal share of
    all steps, made larger by an eighth until they fit into whole rounds of the machine."""
    room = PLACES * (1 + (4 * len(units) + PLACES) // (4 * PLACES))
    size = max(LEAST, -(-sum(units) // room))
    while True:
        parts = [-(-n // size) for n in units]
        if sum(parts) <= room:
            return sum(parts), sum(k for k in parts if k > 1)
        size += (size >> 3) + 1


def test_parts_that_leave_partial_results():
    rng = random.Random(1)
    worst = 0
    for _ in range(4000):
        n, long = rng.randint(1, 2000), rng.randint(1, 3000)
        worst = max(worst, cut([rng.choice([1, long, rng.randint(1, long)]) for _ in range(n)])[1])
    assert worst <= MOST
    assert cut([100] * 320 + [1] * 128) == (768, 640)             # the most there can be


def query(T, heads, latent, rope=64, max_fresh=None, n_requests=4, max_length=9000):
    cache = G.make_latent_cache(codes=0, scales=0, ropes=0, n_blocks=1 << 16, block_tokens=64, latent_dim=latent, rope_dim=rope, act_dtype=G.GLOWQ_BF16)
    return G.glowq_latent_attention_workspace_bytes(cache, G.make_latent_attention(
        q=0, out=0, table=0, lengths=0, starts=0, ldq=heads * (latent + rope), ldo=heads * latent, table_width=1 << 12, n_requests=n_requests, T=T, heads=heads,
        max_fresh=T if max_fresh is None else max_fresh, max_length=max_length, scale=0.1))


@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("heads", [1, 16, 40, 128])
def test_sizes(heads, latent):
    # 64 rows of sums, references and sums of weights, and a ticket, for each
    most = MOST * (64 * (latent + 2) * 4 + 64)
    sizes = [query(T, heads, latent) for T in (1, 7, 100, 2048, 8192, 1 << 20)]
    assert max(sizes) <= most and sizes == sorted(sizes)
    # a part of two steps leaves none
    assert query(1, heads, latent, max_length=128) == 256


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_as_many_partial_results_as_there_can_be(act):
    rng = np.random.default_rng(4)
    b = Absorbed(rng, [(100 * STEP - 1, 1)], 5, 256, 32, 128, act)
    b.fresh, b.lengths = [1] * 448, [int(v) for v in rng.permutation([100 * STEP] * 320 + [STEP] * 128)]
    b.starts, b.T, b.table = np.arange(449), 449, np.repeat(b.table, 448, 0)
    b.q = np.repeat(b.q[:1], 449, 0)
    b.device()
    need = b.ws.numel()
    assert need == MOST * (16 * 258 * 4 + 64)
    mem = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    b.ws = mem[:need]
    out = b.run().output()
    assert (mem[need:] == 0xFF).all(), "written behind the workspace"
    long = np.array(b.lengths) > STEP
    assert (out[long] == out[long][0]).all() and (out[~long] == out[~long][0]).all()
    lengths = b.lengths
    b.fresh = [int(i in (int(long.argmax()), int((~long).argmax()))) for i in range(448)]          # the reference takes its time
    want, bound = b.reference()
    for i in np.flatnonzero(b.fresh):
        assert (np.abs(out[i] - want[i]) <= bound[i]).all(), (i, lengths[i])


@pytest.mark.gpu
def test_a_long_piece_of_many_tiles():
    # 1100 units of 64 rows, those of the first request with many more keys than the others
    rng = np.random.default_rng(5)
    b = Absorbed(rng, [(9000, 5), (0, 500), (0, 45)], 128, 256, 32, 64, "bf16")
    first = b.device().run().check()
    assert b.ws.numel() == MOST * (64 * 258 * 4 + 64)
    assert np.array_equal(first, b.run().output())
