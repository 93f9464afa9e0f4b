"""Attention over the 8-bit cache where memory holds anything, scales lie far apart, or a caller's bounds are smaller than
what a call brings: outputs against the definition in 64 bits, within what rounding the weights allows."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as K
from kv_util import ROUNDOFF, Batch

pytestmark = pytest.mark.gpu


def contract(b, cap=None):
    """(out, bound) in 64 bits for every row, keys from `cap` on left out.  The bound, with u the roundoff of the activation type:
    a weight is rounded once, off by u of itself and in binary16 by 2^-25 of the row's largest, in the product with V and in
    the sum of weights; scores in fp32 are off by (D + 4) 2^-24 sum |q k| scale, and so are a weight and their sum; sums over L
    keys and the exponential's last places; the result's own rounding.  No term goes by another block's magnitude."""
    u, group, D = ROUNDOFF[b.act], b.heads // b.kv, b.D
    least, tiny = (2.0 ** -25, 2.0 ** -24) if b.act == "f16" else (0.0, 1e-38)
    out, bound = np.zeros((int(b.starts[-1]), b.heads, D)), np.zeros((int(b.starts[-1]), b.heads, D))
    for r, L in enumerate(b.lengths):
        f, n = b.fresh[r], max(L, 0) if cap is None else max(min(L, cap), 0)
        if f == 0 or n == 0:
            continue
        j = np.arange(n)
        e = np.where(j // b.B < b.table.shape[1], b.table[r][np.minimum(j // b.B, b.table.shape[1] - 1)], -1)
        there = (e >= 0) & (e < b.cache.n_blocks)
        slots = np.where(there, e * b.B + j % b.B, -1)
        Kt, Vt = (torch.from_numpy(b.cache.tokens(w, slots)).cuda() for w in range(2))
        qr = torch.from_numpy(b.q[int(b.starts[r]):int(b.starts[r]) + f]).cuda()
        p, j = torch.arange(L - f, L, device="cuda")[:qr.shape[0], None], torch.from_numpy(j).cuda()[None]
        see = (j <= p) & torch.from_numpy(there).cuda()[None]
        if b.window:
            see &= j > p - b.window
        none, seen = ~see.any(1), see.double()
        for h in range(b.heads):
            k, v, rows = Kt[:, h // group].contiguous(), Vt[:, h // group].contiguous(), qr[:, h].contiguous()
            w = torch.softmax((rows @ k.T.contiguous() * b.scale).masked_fill(~see, -math.inf), 1)
            w[none] = 0.0
            size = (rows.abs() @ k.abs().T.contiguous() * b.scale * seen).amax(1, keepdim=True)
            o, mag = w @ v, w @ v.abs()
            eps = 2.0 ** -24 * (2 * (D + 4) * size + 2 * n + 64)
            small = least * w.amax(1, keepdim=True) * (seen @ v.abs() + seen.sum(1, keepdim=True) * o.abs())
            t = slice(int(b.starts[r]), int(b.starts[r]) + qr.shape[0])
            out[t, h] = o.cpu().numpy()
            bound[t, h] = ((1 + 4 * u) * ((u + eps) * (mag + o.abs()) + small + u * o.abs()) + tiny).cpu().numpy()
    return out, bound


def agree(got, out, bound):
    bad = ~(np.abs(got - out) <= bound)
    assert not bad.any(), (int(bad.sum()), bad.size, float(np.nanmax(np.abs(got - out) / bound)), np.argwhere(bad)[:4].tolist())


def unused_blocks(b):
    return np.setdiff1d(np.arange(b.cache.n_blocks), b.table[b.table >= 0])


def without_block_0(b):
    """No request has block 0 (what was in it moves to a block that no request has)."""
    b.table[b.table == 0] = unused_blocks(b)[-1]
    b.used = [int(b.table[r, j // b.B]) * b.B + j % b.B for r, L in enumerate(b.lengths) for j in range(max(L, 0)) if b.table[r, j // b.B] >= 0]
    return b


def fill_unused_scales(b, byte):
    at = torch.from_numpy(unused_blocks(b)).cuda()
    for s in b.dc.scales:
        s[at] = byte
    return b


# few rows, many, both; what lies behind the last key ends anywhere in a tile
SHAPES = {"few": [(0, 1), (4, 1), (15, 1), (16, 1), (31, 1), (32, 1), (47, 1), (111, 1), (140, 1)],
          "many": [(0, 40), (13, 70), (100, 129)], "both": [(36, 1), (0, 49), (3, 1), (66, 33), (20, 2)]}


# ---- memory that nobody wrote ---------------------------------------------------------------
@pytest.mark.parametrize("byte", [0, 255])
@pytest.mark.parametrize("act,heads,kv,D,B", [("f16", 8, 2, 128, 64), ("bf16", 4, 4, 64, 16), ("bf16", 8, 2, 128, 16), ("f16", 4, 1, 64, 32)])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scales_of_blocks_that_no_request_has(shape, act, heads, kv, D, B, byte):
    b = without_block_0(Batch(np.random.default_rng(40), SHAPES[shape], heads, kv, D, B, act))
    fill_unused_scales(b.device(), byte).run()
    agree(b.output(), *contract(b))


@pytest.mark.parametrize("byte", [0, 255])
@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("requests", [[(150, 1), (70, 1)], [(60, 40), (90, 50)]])
def test_scales_where_blocks_are_not_there(requests, act, byte):
    b = Batch(np.random.default_rng(41), requests, 4, 2, 64, 16, act)
    b.table[0, 1], b.table[0, 3], b.table[1, 0], b.table[1, 4] = -1, b.cache.n_blocks, -1, 1 << 30
    without_block_0(b)
    fill_unused_scales(b.device(), byte).run()
    agree(b.output(), *contract(b))


@pytest.mark.parametrize("byte", [0, 255])
@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("requests,window", [([(99, 1), (86, 1)], 20), ([(60, 40), (90, 50)], 25)])
def test_blocks_before_the_window_may_be_given_back(requests, window, act, byte):
    """Entries of blocks that the window has left behind name a block that nobody wrote."""
    b = Batch(np.random.default_rng(42), requests, 4, 2, 64, 16, act)
    without_block_0(b)
    for r, (c, _) in enumerate(requests):
        b.table[r, :max(0, c - window + 1) // 16] = 0
    used = [int(b.table[r, j // 16]) * 16 + j % 16 for r, L in enumerate(b.lengths) for j in range(L)]
    b.used = [s for s in used if s >= 16]
    b.device(window=window)
    for s in b.dc.scales:
        s[0] = byte
    b.run()
    agree(b.output(), *contract(b))


# ---- scales far apart ---------------------------------------------------------------------
@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("order", ["01", "10", "010", "101", "0011", "1100", "00001", "1000010"])
@pytest.mark.parametrize("single", [True, False])
def test_a_block_of_zeros_keeps_its_weight(act, D, order, single):
    """Equal scores: the mean of the values seen, blocks of zeros (the smallest exponent) and of ones."""
    L = 16 * len(order)
    fresh = 1 if single else L
    b = Batch(np.random.default_rng(43), [(L - fresh, fresh)], 4, 1, D, 16, act)
    for i, c in enumerate(order):
        at = int(b.table[0, i])
        b.cache.codes[1][at], b.cache.exps[1][at] = (0, K.EXP_MIN) if c == "0" else (K.encode(np.array(256.0)), -8)
    b.q[:] = 0.0
    b.device().run()
    ones = np.repeat([c == "1" for c in order], 16)
    want = (np.cumsum(ones) / np.arange(1, L + 1))[L - fresh:, None, None]
    got = b.output()
    # (weights of one: sums are exact, one division and one rounding)
    assert (np.abs(got - want) <= 1.01 * ROUNDOFF[act] * want).all(), float(np.abs(got - want).max())


FAR = [([(31, 1), (95, 1), (300, 1)], 4, 1), ([(0, 32), (20, 100), (260, 40)], 4, 2), ([(500, 1), (40, 60)], 8, 2)]


@pytest.mark.parametrize("act,D,B", [("f16", 128, 16), ("f16", 64, 16), ("f16", 128, 32), ("bf16", 128, 16)])
@pytest.mark.parametrize("requests,heads,kv", FAR)
@pytest.mark.parametrize("apart", [8, 14, 15, 16, 20, 23, 24, 30])
def test_values_of_blocks_far_apart(act, D, B, requests, heads, kv, apart):
    """Neighbouring blocks of a request 2^apart apart, in either order."""
    b = Batch(np.random.default_rng(44 + apart), requests, heads, kv, D, B, act, q_scale=2.0)
    for r in range(len(requests)):
        for i, at in enumerate(b.table[r]):
            if at >= 0:
                b.cache.exps[1][at] = 4 - (apart if (i + r) % 2 else 0)
    b.device().run()
    agree(b.output(), *contract(b))


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("requests,heads,kv", FAR)
@pytest.mark.parametrize("gap", [-26.0, -8.0, 8.0])
def test_one_block_far_larger(act, requests, heads, kv, gap):
    """One block 2^14 larger than the rest, whose keys score far below them or far above."""
    b = Batch(np.random.default_rng(46), requests, heads, kv, 64, 16, act, q_scale=0.2)
    b.cache.exps[1][:] = -8
    b.cache.exps[0][:] = -4
    b.cache.codes[0][..., 0] = 0
    b.q[..., 0] = 8.0
    for r in range(len(requests)):
        at = int(b.table[r, 1])
        b.cache.exps[1][at] = 6
        b.cache.codes[0][at, ..., 0] = K.encode(np.array(gap * 2.0 ** 4))          # 8 of q, 1 / 8 of the scores' scale
    b.device().run()
    agree(b.output(), *contract(b))


@pytest.mark.parametrize("act,low,high", [("f16", -30, 7), ("f16", -64, 7), ("bf16", -64, 20), ("bf16", -64, 119)])
@pytest.mark.parametrize("requests", [[(9000, 1)], [(4000, 60)], [(2500, 1), (700, 33), (0, 1), (1200, 2)], [(0, 300)]])
@pytest.mark.parametrize("D,B", [(128, 16), (64, 64)])
def test_value_scales_at_random(act, low, high, requests, D, B):
    """Every block its own, in calls that are cut and joined too."""
    rng = np.random.default_rng(47)
    b = Batch(rng, requests, 8, 2, D, B, act)
    b.cache.exps[1][:] = rng.integers(low, high + 1, b.cache.exps[1].shape)
    b.cache.exps[1][rng.random(b.cache.exps[1].shape) < 0.3] = K.EXP_MIN
    b.cache.codes[1][b.cache.exps[1] == K.EXP_MIN] = 0
    first = b.device().run().output()
    agree(first, *contract(b))
    b.dout.fill_(float("nan"))
    assert np.array_equal(b.run().output(), first)


# ---- scales of the scores --------------------------------------------------------------------
@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1e-20, 1e-30, 1e-38, 1e-42])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scores_next_to_nothing(shape, scale, act):
    """Key scale times score scale under the range of fp32: flat weights, and hidden keys hidden."""
    b = Batch(np.random.default_rng(56), SHAPES[shape], 4, 2, 64, 16, act)
    b.cache.exps[0][:] = K.EXP_MIN
    b.device(scale=scale).run()
    agree(b.output(), *contract(b))


# ---- bounds smaller than what a call brings --------------------------------------------------
@pytest.mark.parametrize("heads,kv,max_fresh", [(4, 1, 4), (4, 2, 4), (8, 1, 7), (2, 2, 1), (4, 1, 33)])
@pytest.mark.parametrize("window", [0, 20])
def test_rows_past_max_fresh_are_left_out(heads, kv, max_fresh, window):
    """The rows before them keep their positions."""
    b = Batch(np.random.default_rng(50), [(50, 10), (20, 3), (0, 60), (7, 1)], heads, kv, 64, 16, "f16")
    b.device(max_fresh=max_fresh, window=window).run()
    got, (out, bound) = b.output(), contract(b)
    for r, f in enumerate(b.fresh):
        at, kept = int(b.starts[r]), min(f, max_fresh)
        agree(got[at:at + kept], out[at:at + kept], bound[at:at + kept])
        assert np.isnan(got[at + kept:at + f]).all()


@pytest.mark.parametrize("requests", [[(50, 10), (20, 9)], [(33, 1), (5, 70)], [(0, 4), (60, 2), (9, 5)]])
def test_rows_past_those_that_q_holds_are_left_out(requests):
    b = Batch(np.random.default_rng(51), requests, 4, 2, 64, 16, "bf16", extra_rows=-4)
    b.device(max_fresh=min(b.T, max(b.fresh))).run()
    torch.cuda.synchronize()
    got, (out, bound) = b.dout.double().cpu().numpy().reshape(b.T, 4, 64), contract(b)
    agree(got, out[:b.T], bound[:b.T])


@pytest.mark.parametrize("requests", [[(99, 1)], [(70, 30)], [(40, 60), (99, 1)]])
def test_windows_past_max_length_hide_keys_all_the_same(requests):
    """A window as long as the bound of lengths, on requests that are longer: keys past the bound are left out, and so are those
    before the window."""
    b = Batch(np.random.default_rng(52), requests, 4, 2, 64, 16, "f16")
    b.device(max_length=50, window=60).run()
    agree(b.output(), *contract(b, cap=50))


# ---- rows that see no key -------------------------------------------------------------------
@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("requests,window", [([(30, 1), (40, 1)], 0), ([(30, 20), (40, 33)], 0), ([(30, 1), (200, 1), (0, 50)], 24), ([(3000, 1), (40, 1)], 0),
                                             ([(1500, 40), (40, 3)], 0)])
def test_rows_whose_blocks_are_all_outside_the_cache_are_zeros(act, requests, window):
    b = Batch(np.random.default_rng(53), requests, 4, 2, 64, 16, act)
    b.table[0] = -1
    b.table[0, ::3] = b.cache.n_blocks
    if window:
        b.table[1, 10:] = -1                                        # (the window's only)
    got = b.device(window=window).run().output()
    assert (got[:int(b.starts[1])] == 0).all()
    agree(got, *contract(b))


@pytest.mark.parametrize("fresh", [1, 40])
def test_rows_whose_scores_are_all_minus_infinity_are_no_numbers(fresh):
    b = Batch(np.random.default_rng(54), [(20, fresh), (20, 1)], 4, 2, 64, 16, "f16")
    b.cache.codes[0][:] = K.encode(np.array(64.0))
    b.q[:fresh] = -np.inf
    got = b.device().run().output()
    assert np.isnan(got[:fresh]).all() and not np.isnan(got[fresh:]).any()


# ---- lengths far past the table --------------------------------------------------------------
@pytest.mark.parametrize("heads,fresh", [(2, 1), (8, 9), (4, 40)])
@pytest.mark.parametrize("length", [1 << 20, (1 << 30) + 5, (1 << 31) - 4000, (1 << 31) - 1])
@pytest.mark.parametrize("window", [0, 1, 20])
def test_lengths_far_past_the_table(heads, fresh, length, window):
    """Keys past max_length and the table's width are left out: under a window nothing is left, without one what is there."""
    b = Batch(np.random.default_rng(55), [(64 - fresh, fresh), (30, 1)], heads, 2, 64, 16, "f16")
    b.device(max_length=64, window=window)
    b.dlengths[0] = length
    got = b.run().output()
    b.lengths[0] = 64 + fresh - 1                                   # (every row sees all keys of the table)
    out, bound = contract(b, cap=64)
    if window:
        out[:fresh] = bound[:fresh] = 0.0
    agree(got, out, bound)


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,requests", [(2, [(60, 7), (90, 5), (1500, 4)]), (8, [(50, 40), (0, 90), (1300, 70)])])
def test_hidden_numbers_that_are_none_where_scales_lie_far_apart(heads, requests, D, act):
    """A value that is none, in a tile of blocks 2^24 apart: rows in front of it are what they are without it, those behind have it."""
    b = Batch(np.random.default_rng(57), requests, heads, 2, D, 16, act)
    for r in range(len(requests)):
        for i, at in enumerate(b.table[r]):
            if at >= 0:
                b.cache.exps[1][at] = (3, -21, K.EXP_MIN)[(i + r) % 3]
                if (i + r) % 3 == 2:
                    b.cache.codes[1][at] = 0
    group, spoilt, early = heads // 2, [], np.zeros((int(b.starts[-1]), heads), bool)
    for r, (c, f) in enumerate(requests):
        at = c + f // 2
        slot = int(b.table[r, at // 16]) * 16 + at % 16
        spoilt.append((slot // 16, 1, slot % 16, 9))
        early[int(b.starts[r]):int(b.starts[r]) + f // 2] = True
    early[:, :group] = True
    kept = [b.cache.codes[1][at] for at in spoilt]
    for at in spoilt:
        b.cache.codes[1][at] = K.NAN_CODE
    got = b.device().run().output()
    for at, code in zip(spoilt, kept):
        b.cache.codes[1][at] = code
    out, bound = contract(b)
    agree(got[early], out[early], bound[early])
    want = np.zeros(got.shape, bool)
    want[..., 9] = ~early
    assert np.array_equal(np.isnan(got), want)
    rest = ~early[..., None] & ~want
    agree(got[rest], out[rest], bound[rest])
