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
