"""GPU parity of rotary positions with their oracle: rows in memory, keys on their way into the 8-bit cache."""
import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from gpu_util import ACT_CODE, TORCH_ACT, stream
from kv_util import DeviceCache, act_round, i32, random_cache
from latent_util import ROUNDOFF, TINY, Rope, Rows, rope_rows

pytestmark = pytest.mark.gpu


def numbers(rng, T, h, d, act):
    x = rng.standard_normal((T, h, d)) * 2
    return act_round(x, act) if act != "f32" else x.astype(np.float32).astype(np.float64)


def check_rotated(rope, x, got, positions, act):
    want = rope.rotate(x, positions)
    live = np.asarray(positions) >= 0
    bound = rope.slack(x) + ROUNDOFF[act] * np.abs(want) + TINY[act]
    bound[..., rope.r:] = 0.0                                     # the rest is as it was
    off = np.abs(got - want)[live]
    assert (off <= bound[live]).all(), float(np.nanmax(off / np.maximum(bound[live], 1e-300)))


@pytest.mark.parametrize("act", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("T,heads,D,r,gap,pad", [(1, (1, 1), 16, 16, 0, 0), (5, (3, 2), 64, 32, 8, 0), (67, (8, 1), 128, 128, 0, 8), (200, (7, 3), 96, 48, 16, 24),
                                                 (2100, (32, 8), 128, 64, 0, 0), (33, (5, 5), 256, 256, 0, 0)])
def test_rows(act, layout, T, heads, D, r, gap, pad):
    rng = np.random.default_rng(T)
    rope = Rope(r, layout, ["plain", "ramp", "bands"][T % 3])
    positions = rng.integers(0, 1 << 17, T)
    positions[rng.random(T) < 0.2] = -1
    positions[:1] = (1 << 31) - 1                                 # the farthest of all
    xs = [numbers(rng, T, h, D, act) for h in heads]
    ins, outs = [Rows(x, act, gap, pad) for x in xs], [Rows(np.zeros_like(x), act, 8, 16, filled=False) for x in xs]
    at = i32(positions)
    G.glowq_rotate(rope.desc, [rope_rows(i, o) for i, o in zip(ins, outs)], D, ACT_CODE[act], at.data_ptr(), T, stream())
    for x, i, o in zip(xs, ins, outs):
        got = o.numbers()
        assert np.isnan(got[positions < 0]).all(), "rows without a position were written"
        check_rotated(rope, x, got, positions, act)
        assert np.array_equal(i.numbers(), x)
    # in place: the same bits, rows without a position as they were
    G.glowq_rotate(rope.desc, [rope_rows(i, i) for i in ins], D, ACT_CODE[act], at.data_ptr(), T, stream())
    for x, i, o in zip(xs, ins, outs):
        got, want = i.numbers(), o.numbers()
        assert np.array_equal(got[positions >= 0], want[positions >= 0]) and np.array_equal(got[positions < 0], x[positions < 0])


def test_four_tensors_and_numbers_that_are_none():
    rng = np.random.default_rng(4)
    rope, T = Rope(32, "pairs"), 9
    positions = np.arange(T) * 1000
    xs = [numbers(rng, T, h, 48, "bf16") for h in (1, 2, 3, 4)]
    xs[2][3, 1, 5], xs[2][4, 2, 40] = np.inf, np.nan
    rows, at = [Rows(x, "bf16") for x in xs], i32(positions)
    G.glowq_rotate(rope.desc, [rope_rows(i, i) for i in rows], 48, G.GLOWQ_BF16, at.data_ptr(), T, stream())
    for k, (x, i) in enumerate(zip(xs, rows)):
        got = i.numbers()
        if k == 2:
            # dims 4 and 5 are a pair; nothing else knows of them
            assert not np.isfinite(got[3, 1, 4:6]).any() and np.isnan(got[4, 2, 40])
            got[3, 1, 4:6], x[3, 1, 4:6], got[4, 2, 40], x[4, 2, 40] = 0.0, 0.0, 0.0, 0.0
        check_rotated(rope, x, got, positions, "bf16")


def append_rotated(dc, rope, q, rows, slots, positions, act, pad=0):
    w = dc.o.kv * dc.o.D
    dev = [Rows(x, act, 0, pad) for x in rows]
    out = None if q is None else Rows(np.zeros_like(q), act, 8, 0, filled=False)
    dslots, dpositions = i32(slots), i32(positions)
    dq = None if q is None else Rows(q, act)
    G.glowq_kv_append_rotated(dc.desc, rope.desc, None if q is None else rope_rows(dq, out), dev[0].buf.data_ptr(), w + pad, dev[1].buf.data_ptr(), w + pad,
                              ACT_CODE[act], dslots.data_ptr(), dpositions.data_ptr(), len(slots), stream())
    torch.cuda.synchronize()
    return None if q is None else out.numbers()


def check_rotated_cache(dc, held):
    """Values as the oracle's; keys on the grid of the block's exponent, nearest to the rotated numbers up to the error of those.  held:
    slot -> (rotated key, its slack)."""
    c = dc.o
    slots = np.array(sorted(held))
    assert np.array_equal(dc.tokens(1, slots), c.tokens(1, slots), equal_nan=True)
    got, want = dc.tokens(0, slots), c.tokens(0, slots)
    assert np.array_equal(dc.scales[0].cpu().numpy()[slots // c.B], (c.exps[0] + 127).astype(np.uint8)[slots // c.B])
    x, slack = (np.stack([held[s][i] for s in slots]) for i in range(2))
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = (got == want) | np.isnan(want) | (np.abs(got - x) <= np.abs(want - x) + slack)
    assert ok.all() and (got != want)[~np.isnan(want)].mean() < 1e-3


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("B,kv,D,r,layout", [(16, 1, 64, 64, "halves"), (32, 3, 128, 64, "pairs"), (64, 9, 64, 32, "halves"), (128, 6, 128, 128, "pairs")])
def test_keys_on_their_way_into_the_cache(act, B, kv, D, r, layout):
    rng = np.random.default_rng(B + D)
    dc, rope = DeviceCache(random_cache(rng, 12, B, kv, D), used=[]), Rope(r, layout, "ramp")
    order = rng.permutation(12)
    a, b = order[:5], order[5:9]
    slot = lambda blocks, j: blocks[j // B] * B + j % B
    na, nb = 2 * B + 5, B - 1
    pieces = [(np.concatenate([slot(a, np.arange(na)), slot(b, np.arange(nb))]), np.concatenate([np.arange(na), 70000 + np.arange(nb)]), 1.0)]
    for k in range(4):
        pieces.append((np.array([slot(a, na + k), slot(b, nb + k)]), np.array([na + k, 70000 + nb + k]), [0.3, 5.0, 40.0, 0.01][k]))
    pieces.append((slot(a, np.arange(na + 4, 4 * B + 1)), np.arange(na + 4, 4 * B + 1), 2.0))
    held, exps = {}, {}
    for k, (slots, positions, size) in enumerate(pieces):
        T = len(slots)
        q = numbers(rng, T, 4, D, act)
        rows = [act_round(rng.standard_normal((T, kv, D)) * size, act) for _ in range(2)]
        turned = rope.rotate(rows[0], positions)
        slack = rope.slack(rows[0])
        dc.o.append([turned, rows[1]], slots)
        got = append_rotated(dc, rope, q, rows, slots, positions, act, pad=8 * (k % 3))
        check_rotated(rope, q, got, positions, act)
        # older tokens of a block that grew are on another grid than they were rounded to at first: what they were then is what counts
        for i, s in enumerate(slots):
            held[int(s)] = (turned[i], slack[i])
        for s in held:
            old = exps.get(s)
            now = dc.o.exps[0][s // B].copy()
            if old is not None and (old != now).any():
                del_now = dc.o.tokens(0, [s])[0]
                held[s] = (del_now, held[s][1] + np.ldexp(1.0, now)[:, None] * 64)        # a step of the new grid at most
            exps[s] = now
        check_rotated_cache(dc, held)


def test_many_rows_and_some_without_a_slot():
    rng = np.random.default_rng(8)
    T, B, kv = 4321, 32, 5
    dc, rope = DeviceCache(random_cache(rng, 400, B, kv, 64), used=[]), Rope(64)
    order, slots, positions, block = rng.permutation(400), [], [], 0
    while len(slots) < T and block < 390:
        f, lo = int(rng.choice([1, 1, 2, 7, 31, 32, 33, 100])), int(rng.integers(0, B))
        for j in range(lo, lo + f):
            slots.append(order[block + j // B] * B + j % B)
            positions.append(5 * block + j)
        block += (lo + f - 1) // B + 1
    slots, positions = np.array(slots), np.array(positions)
    positions[7] = -5                                             # counts as 0 for a key that has a slot; q's row stays
    gone = rng.random(len(slots)) < 0.02
    gone[7] = False
    slots[gone], n = -1, len(slots)
    slots[np.flatnonzero(gone)[:2]] = (400 * B, 1 << 30)          # behind the cache
    # (the rows of a block are to be neighbours: those behind a gap are left out too)
    broken = {}
    for t in range(n):
        if 0 <= slots[t] < 400 * B and broken.setdefault(slots[t] // B, slots[t]) != slots[t]:
            slots[t] = -1
        elif 0 <= slots[t] < 400 * B:
            broken[slots[t] // B] = slots[t] + 1
    rows = [act_round(rng.standard_normal((n, kv, 64)), "f16") for _ in range(2)]
    at = np.maximum(positions, 0)
    turned, slack = rope.rotate(rows[0], at), rope.slack(rows[0])
    before = {w: dc.tokens(w, np.arange(400 * B)) for w in range(2)}
    dc.o.append([turned, rows[1]], slots)
    q = numbers(rng, n, 3, 64, "f16")
    got = append_rotated(dc, rope, q, rows, slots, positions, "f16")
    assert np.isnan(got[7]).all()
    check_rotated(rope, q, got, positions, "f16")
    there = (slots >= 0) & (slots < 400 * B)
    check_rotated_cache(dc, {int(s): (turned[i], slack[i]) for i, s in enumerate(slots) if there[i]})
    touched = np.unique(slots[there] // B)
    rest = np.setdiff1d(np.arange(400), touched)
    for w in range(2):
        now = dc.tokens(w, np.arange(400 * B)).reshape(400, B, kv, 64)
        assert np.array_equal(now[rest], before[w].reshape(400, B, kv, 64)[rest], equal_nan=True)


@pytest.mark.parametrize("act", ["f16", "bf16"])
def test_keys_that_are_no_numbers(act):
    rng = np.random.default_rng(3)
    dc, rope = DeviceCache(random_cache(rng, 4, 16, 2, 64), used=[]), Rope(32, "pairs")
    slots, positions = np.arange(16, 26), np.arange(100, 110)
    rows = [act_round(rng.standard_normal((10, 2, 64)), act) for _ in range(2)]
    rows[0][2, 0, 4], rows[0][3, 1, 50], rows[1][5, 1, 7] = np.inf, np.nan, -np.inf
    turned = rope.rotate(np.where(np.isfinite(rows[0]), rows[0], 0.0), positions)
    turned[2, 0, 4:6], turned[3, 1, 50] = np.nan, np.nan           # the pair of an infinity is not finite
    dc.o.append([turned, rows[1]], slots)
    append_rotated(dc, rope, None, rows, slots, positions, act)
    slack = rope.slack(np.where(np.isfinite(rows[0]), rows[0], 0.0))
    check_rotated_cache(dc, {int(s): (turned[i], slack[i]) for i, s in enumerate(slots)})


def test_a_rotation_in_a_graph_is_replayed():
    rng = np.random.default_rng(5)
    rope, x = Rope(64), numbers(rng, 50, 6, 64, "bf16")
    dc = DeviceCache(random_cache(rng, 8, 64, 2, 64), used=[])
    i, o, positions, slots = Rows(x, "bf16"), Rows(np.zeros_like(x), "bf16", filled=False), i32(np.arange(50)), i32(np.arange(64, 114))
    k, v = Rows(x[:, :2], "bf16"), Rows(x[:, 2:4], "bf16")

    def call(st):
        G.glowq_rotate(rope.desc, [rope_rows(i, o)], 64, G.GLOWQ_BF16, positions.data_ptr(), 50, st)
        G.glowq_kv_append_rotated(dc.desc, rope.desc, None, k.buf.data_ptr(), 128, v.buf.data_ptr(), 128, G.GLOWQ_BF16, slots.data_ptr(), positions.data_ptr(), 50, st)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(side.cuda_stream)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(side.cuda_stream)
    for n in range(3):
        positions.copy_(i32(np.arange(50) * (n + 1)))
        x = numbers(rng, 50, 6, 64, "bf16")
        i.view[:] = torch.from_numpy(x).to(torch.bfloat16).cuda()
        k.view[:] = i.view[:, :2]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check_rotated(rope, x, o.numbers(), np.arange(50) * (n + 1), "bf16")
        replayed = dc.codes[0].clone()
        dc.codes[0].fill_(0xFF)                                       # as the cache was made
        call(stream())
        torch.cuda.synchronize()
        assert torch.equal(replayed, dc.codes[0])
