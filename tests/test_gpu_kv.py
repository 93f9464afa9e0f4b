"""GPU parity of the serving operators with their oracle: tables and slots equal, the cache's bytes equal, attention within
the bound that its roundings allow (tests/kv_util.py derives it)."""
import math

import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from gpu_util import ACT_CODE, TORCH_ACT, stream
from kv_util import Batch, DeviceCache, act_round, i32, random_cache

pytestmark = pytest.mark.gpu


# ---- tables and slots ---------------------------------------------------------------------
def run_plan(cached, fresh, free, table, B, max_tokens):
    n = len(cached)
    d = dict(cached=i32(cached), fresh=i32(fresh), free_blocks=i32(free if len(free) else [0]), table=i32(table),
             lengths=i32([-9] * n), starts=i32([-9] * (n + 1)), slots=i32([-9] * (max_tokens + 4)),
             positions=i32([-9] * (max_tokens + 4)), taken=i32([-9, -9]))
    s = G.make_kv_step(**{k: v.data_ptr() for k, v in d.items()}, n_requests=n, n_free=len(free), table_width=table.shape[1],
                       max_tokens=max_tokens, block_tokens=B)
    for _ in range(2):                                            # the same call again writes the same
        G.glowq_kv_plan(s, stream())
    torch.cuda.synchronize()
    assert (d["slots"][max_tokens:] == -9).all() and (d["positions"][max_tokens:] == -9).all() and d["taken"][1] == -9
    return d


def check_plan(cached, fresh, free, table, B, max_tokens):
    want = np.array(table)
    lengths, starts, slots, positions, taken = K.plan(cached, fresh, free, want, B, max_tokens)
    d = run_plan(cached, fresh, free, table, B, max_tokens)
    for name, v in (("lengths", lengths), ("starts", starts), ("slots", slots), ("positions", positions), ("table", want)):
        assert np.array_equal(d[name].cpu().numpy()[..., :v.shape[-1]], v), name
    assert int(d["taken"][0]) == taken


@pytest.mark.parametrize("n,B,pad", [(1, 16, 0), (3, 64, 5), (64, 32, 0), (255, 16, 1), (257, 128, 100), (1500, 16, 0), (9001, 16, 7)])
def test_plan(n, B, pad):
    rng = np.random.default_rng(n)
    cached = rng.integers(0, 5 * B, n)
    fresh = np.where(rng.random(n) < 0.5, 1, rng.integers(0, 3 * B + 2, n))
    cached[rng.random(n) < 0.2] = 0
    had = -(-cached // B)
    width = int(max(1, (-(-(cached + fresh) // B)).max())) + 1
    ids = rng.permutation(int(had.sum()) + int((-(-(cached + fresh) // B) - had).sum()) + 5)
    table, at = np.full((n, width), -1), 0
    for r in range(n):
        table[r, :had[r]] = ids[at:at + had[r]]
        at += had[r]
    check_plan(cached, fresh, ids[at:], table, B, max(1, int(fresh.sum()) + pad))


def test_plan_where_something_runs_out():
    table = np.full((4, 3), -1)
    table[0, 0], table[1, :2] = 5, (1, -1)
    check_plan([10, 20, 0, 0], [30, 2, 0, 20], [7, 3], table, 16, 60)                 # blocks: two of five are there
    check_plan([10, 20, 0, 0], [30, 2, 0, 20], [], table, 16, 60)                     # none
    check_plan([10, 20, 0, 0], [90, 2, 0, 20], list(range(20)), table, 16, 200)       # the table's width
    check_plan([10, -3, 0, 0], [30, 2, -5, 20], list(range(20)), table, 16, 60)       # negative numbers count as none
    check_plan([0, 0, 0, 0], [0, 0, 0, 0], [2], table, 16, 3)                         # nothing to do
    check_plan([10, 20, 0, 0], [30, 2, 0, 20], list(range(20)), table, 16, 33)        # fewer rows than tokens


# ---- the cache ------------------------------------------------------------------------------
def rows_of(rng, T, kv, D, act, scale=1.0):
    return [act_round(rng.standard_normal((T, kv, D)) * scale, act) for _ in range(2)]


def append(dc, rows, slots, act, pad=0):
    c = dc.o
    T, w = len(slots), c.kv * c.D
    dev = []
    for x in rows:
        t = torch.full((T, w + pad), float("nan"), dtype=TORCH_ACT[act], device="cuda")
        t[:, :w] = torch.from_numpy(x.reshape(T, w)).to(TORCH_ACT[act]).cuda()
        dev.append(t)
    G.glowq_kv_append(dc.desc, dev[0].data_ptr(), w + pad, dev[1].data_ptr(), w + pad, ACT_CODE[act], i32(slots).data_ptr(), T, stream())
    torch.cuda.synchronize()


def check_cache(dc, slots):
    """Bytes of these tokens, and their blocks' scales, as the oracle's."""
    c = dc.o
    for w in range(2):
        codes, scales = c.pages(w)
        at = K.places(c.B, c.D, w == 1)
        dcodes, dscales = dc.codes[w].cpu().numpy(), dc.scales[w].cpu().numpy()
        for s in slots:
            b = int(s) // c.B
            assert np.array_equal(dscales[b], scales[b]), (w, s)
            x, y = K.VALUES[dcodes[b][:, at[int(s) % c.B]]], K.VALUES[codes[b][:, at[int(s) % c.B]]]
            assert np.array_equal(x, y, equal_nan=True), (w, s)


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("B,kv,D", [(16, 1, 64), (32, 3, 128), (64, 2, 64), (128, 2, 128)])
def test_append_prompts_and_single_tokens(act, B, kv, D):
    rng = np.random.default_rng(B + D)
    dc = DeviceCache(random_cache(rng, 12, B, kv, D), used=[])
    order = rng.permutation(12)
    a, b = order[:5], order[5:9]
    slot = lambda blocks, j: blocks[j // B] * B + j % B
    held = []
    # two prompts of odd lengths at once, then tokens one by one with growing and shrinking magnitudes, then a piece that
    # begins within a block
    first = np.concatenate([slot(a, np.arange(2 * B + 5)), slot(b, np.arange(B - 1))])
    pieces = [(first, 1.0)]
    na, nb = 2 * B + 5, B - 1
    for k in range(6):
        pieces.append((np.array([slot(a, na + k), slot(b, nb + k)]), [0.3, 5.0, 1.0, 40.0, 0.01, 1.0][k]))
    pieces.append((slot(a, np.arange(na + 6, 4 * B + 1)), 2.0))
    for k, (slots, scale) in enumerate(pieces):
        rows = rows_of(rng, len(slots), kv, D, act, scale)
        dc.o.append(rows, slots)
        append(dc, rows, slots, act, pad=8 * (k % 3))
        held += list(slots)
        check_cache(dc, held)


def test_append_many_rows_to_a_workgroup():
    # past the number of rows from which a workgroup takes several: runs that begin anywhere in it and go on into the next
    rng = np.random.default_rng(8)
    T, B, kv = 4321, 32, 2
    dc = DeviceCache(random_cache(rng, 400, B, kv, 64), used=[])
    order, slots, block = rng.permutation(400), [], 0
    while len(slots) < T:
        f = int(rng.choice([1, 1, 2, 7, 31, 32, 33, 100]))
        lo = int(rng.integers(0, B))
        for j in range(lo, lo + f):
            slots.append(order[block + j // B] * B + j % B)
        block += (lo + f - 1) // B + 1
        if block > 390:
            break
    slots = np.array(slots)
    slots[rng.random(len(slots)) < 0.02] = -1
    rows = rows_of(rng, len(slots), kv, 64, "f16")
    # (a gap within a block would make two runs of it: the rest of that block's rows are left out too)
    keep = np.ones(len(slots), bool)
    for t in range(1, len(slots)):
        if slots[t] >= 0 and slots[t] % B and not (keep[t - 1] and slots[t - 1] == slots[t] - 1) and slots[t] // B in {
                s // B for s in slots[max(0, t - B):t] if s >= 0}:
            slots[t], keep[t] = -1, False
    assert len(slots) * kv > 8192
    dc.o.append(rows, slots)
    append(dc, rows, slots, "f16")
    check_cache(dc, slots[slots >= 0])


def test_append_numbers_that_are_none_and_extreme_ones():
    rng = np.random.default_rng(9)
    for act, big, tiny in (("f16", 65504.0, 2.0 ** -24), ("bf16", 3.0e38, 1e-38)):
        dc = DeviceCache(random_cache(rng, 6, 32, 2, 64), used=[])
        rows = rows_of(rng, 6 * 32, 2, 64, act)
        for x in rows:
            x[3, 0, 5], x[4, 0, 6], x[5, 1, 7] = np.inf, -np.inf, np.nan      # not part of the scale; stored as NaN
            x[32:64] = 0.0
            x[64:96, 1] = np.nan
            x[96:128] = act_round(x[96:128] * tiny, act)
            x[128:160, 0, :] = act_round(np.clip(x[128:160, 0] * big, -big, big), act)
            x[160:192] = act_round(np.abs(x[160:192]) * 0 + 1.75, act)        # 448 * 2^-8: the boundary of an exponent
            x[161, 1, 3] = act_round(1.7578125, act)
        slots = np.arange(6 * 32)
        dc.o.append(rows, slots)
        append(dc, rows, slots, act)
        check_cache(dc, slots)


def test_slots_outside_the_cache_are_left_out():
    rng = np.random.default_rng(10)
    dc = DeviceCache(random_cache(rng, 3, 16, 1, 64), used=[])
    before = [x.clone() for x in dc.codes + dc.scales]
    append(dc, rows_of(rng, 4, 1, 64, "f16"), [-1, 48, 1 << 30, -16], "f16")
    assert all(torch.equal(x, y) for x, y in zip(before, dc.codes + dc.scales))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_gather(dtype, D):
    rng = np.random.default_rng(11)
    c = random_cache(rng, 7, 32, 3, D)
    c.codes[0][2, 1, 3, 5] = K.NAN_CODE
    c.exps[1][3] = [8, -64, 30 if dtype != "f16" else 0]
    dc = DeviceCache(c)
    slots = rng.permutation(7 * 32)[:150]
    slots[[0, 20]] = -1, 7 * 32
    slots[1] = 2 * 32 + 3
    w = 3 * D
    out = [torch.full((150 + 1, w + 8), 7.0, dtype=TORCH_ACT[dtype], device="cuda") for _ in range(2)]
    G.glowq_kv_gather(dc.desc, i32(slots).data_ptr(), 150, out[0].data_ptr(), w + 8, out[1].data_ptr(), w + 8, ACT_CODE[dtype], stream())
    torch.cuda.synchronize()
    for k in range(2):
        want = torch.from_numpy(c.tokens(k, slots)).float().to(TORCH_ACT[dtype])
        got = out[k][:150, :w].cpu().view(150, 3, D)
        assert torch.equal(torch.nan_to_num(got, nan=123.0), torch.nan_to_num(want, nan=123.0))
        assert (out[k][150] == 7.0).all() and (out[k][:, w:] == 7.0).all()


# ---- attention ------------------------------------------------------------------------------
LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 300]


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,D,B", [(8, 2, 128, 64), (4, 4, 64, 16), (7, 1, 64, 32), (16, 1, 128, 128), (10, 5, 128, 16)])
def test_single_tokens(act, heads, kv, D, B):
    rng = np.random.default_rng(heads * D + B)
    Batch(rng, [(L - 1, 1) for L in LENGTHS], heads, kv, D, B, act, pad_q=8, pad_o=16).device().run().check()


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("heads,kv,D,B", [(8, 2, 128, 64), (4, 4, 64, 16), (7, 1, 64, 32), (20, 1, 128, 32), (6, 6, 128, 128)])
@pytest.mark.parametrize("window", [0, 1, 40, 129])
def test_pieces_and_prompts(act, heads, kv, D, B, window):
    """No tokens, one, several, whole prompts; beside requests without new tokens."""
    rng = np.random.default_rng(heads + D + B + window)
    requests = [(0, 5), (37, 3), (100, 0), (0, 130), (3, 1), (0, 0), (250, 33), (64, 64), (0, 1), (90, 17)]
    Batch(rng, requests, heads, kv, D, B, act, pad_o=8).device(window=window).run().check()


@pytest.mark.parametrize("fresh", [1, 2, 4, 5, 8, 9, 16, 31, 33, 64, 65, 129])
@pytest.mark.parametrize("heads,kv,D", [(4, 1, 128), (3, 3, 64)])
def test_numbers_of_new_tokens(fresh, heads, kv, D):
    rng = np.random.default_rng(fresh)
    Batch(rng, [(111, fresh), (0, fresh), (200, max(1, fresh - 1))], heads, kv, D, 32, "f16").device().run().check()


def test_rows_that_see_nothing_are_zeros():
    rng = np.random.default_rng(20)
    b = Batch(rng, [(-3, 5), (0, 2), (-4, 4), (10, 2)], 4, 2, 64, 16, "f16")      # more new tokens than the length says
    b.device(max_fresh=5, max_length=40).run()
    got = b.check()
    assert (got[:3] == 0).all() and (got[7:11] == 0).all() and not (got[3:7] == 0).all()


def test_hidden_numbers_that_are_none_reach_no_row():
    rng = np.random.default_rng(21)
    for heads, requests in ((4, [(50, 40), (0, 90)]), (2, [(60, 7), (30, 3)])):
        b = Batch(rng, requests, heads, 2, 64, 16, "bf16", pad_q=8)
        want_nan = np.zeros((int(b.starts[-1]), heads, 64), bool)
        for r, (c, f) in enumerate(requests):
            at = c + f // 2                                         # the key in the middle of the new ones
            slot = int(b.table[r, at // 16]) * 16 + at % 16
            for w, head, dim in ((0, 0, 3), (1, 1, 9)):
                b.cache.codes[w][slot // 16, head, slot % 16, dim] = K.NAN_CODE
            t = int(b.starts[r]) + f // 2
            group = heads // 2
            want_nan[t:int(b.starts[r + 1]), :group] = True         # a key: every dim of its heads' rows
            want_nan[t:int(b.starts[r + 1]), group:, 9] = True      # a value: its dim
        b.device().run()
        got = b.output()
        assert np.array_equal(np.isnan(got), want_nan)
        for w in range(2):                                          # the rest is what it is without them
            b.cache.codes[w][b.cache.codes[w] == K.NAN_CODE] = 0
        out, bound = b.reference()
        off = np.abs(got - out)
        early = np.zeros_like(want_nan)
        for r, (c, f) in enumerate(requests):
            early[int(b.starts[r]):int(b.starts[r]) + f // 2] = True
        assert (off[early] <= bound[early]).all()


def test_queries_that_are_no_numbers_stay_in_their_rows():
    rng = np.random.default_rng(22)
    b = Batch(rng, [(70, 1), (20, 9), (5, 1)], 4, 1, 128, 32, "f16")
    clean = b.q.copy()
    bad = [(0, 1), (4, 2), (10, 0)]
    b.q[0, 1, 7], b.q[4, 2, 0], b.q[10, 0, :] = np.inf, np.nan, -np.inf
    b.device().run()
    got = b.output()
    out, bound = b.reference(clean)
    for t, h in bad:
        assert np.isnan(got[t, h]).all()
        got[t, h] = out[t, h]
    assert (np.abs(got - out) <= bound).all()


def test_blocks_outside_the_cache_are_passed_over():
    rng = np.random.default_rng(23)
    b = Batch(rng, [(150, 1), (60, 20)], 4, 2, 64, 16, "f16")
    b.table[0, 2], b.table[0, 9], b.table[1, 0] = -1, b.cache.n_blocks, 1 << 30
    b.device().run().check()


@pytest.mark.parametrize("act", ["f16", "bf16"])
@pytest.mark.parametrize("peak", [0.0, 3.0, 30.0])
def test_scores_far_apart_and_scales_far_apart(act, peak):
    """Flat and sharp scores; blocks whose magnitudes differ by 2^20 in either order."""
    rng = np.random.default_rng(24)
    b = Batch(rng, [(400, 1), (333, 1), (0, 70)], 4, 2, 128, 16, act, q_scale=peak, spread=2)
    n = b.cache.n_blocks
    b.cache.exps[1][:, 0] = rng.integers(-16, 4, n)
    b.device().run().check()


@pytest.mark.parametrize("act,heads,kv,D,B", [("f16", 4, 1, 128, 64), ("bf16", 8, 4, 64, 16)])
@pytest.mark.parametrize("requests,window", [([(9000, 1)], 0), ([(5000, 1), (12, 1), (2500, 1)], 0), ([(6000, 12), (100, 3)], 0),
                                             ([(7000, 1)], 3000), ([(4000, 60)], 0)])
def test_long_contexts_are_cut_and_joined(act, heads, kv, D, B, requests, window):
    rng = np.random.default_rng(25)
    b = Batch(rng, requests, heads, kv, D, B, act).device(window=window)
    first = b.run().check()
    for _ in range(3):                                              # the same bits, through the same workspace
        b.dout.fill_(float("nan"))
        assert np.array_equal(b.run().output(), first)


def test_calls_of_different_sizes_share_a_workspace_on_another_stream_and_in_graphs():
    rng = np.random.default_rng(26)
    batches = [Batch(rng, r, 8, 2, 128, 32, "bf16").device() for r in ([(3000, 1)], [(700, 1)] * 5, [(0, 90), (40, 4)], [(900, 20)])]
    ws = max((b.ws for b in batches), key=lambda t: t.numel())
    G.glowq_workspace_init(ws.data_ptr(), ws.numel(), stream())
    for b in batches:
        b.ws = ws
    want = [b.run().check() for b in batches]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for b in batches:
            b.dout.fill_(float("nan"))
        for b in batches:
            b.run()
        torch.cuda.synchronize()
        for b, w in zip(batches, want):
            assert np.array_equal(b.output(), w)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for b in batches:
                b.run()
        for _ in range(4):
            for b in batches:
                b.dout.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            for b, w in zip(batches, want):
                assert np.array_equal(b.output(), w)
            batches[0].run()                                        # eager work between the replays


def test_many_requests():
    rng = np.random.default_rng(27)
    requests = [(int(rng.integers(0, 60)), int(rng.integers(0, 3))) for _ in range(700)]
    Batch(rng, requests, 4, 2, 64, 16, "f16").device().run().check()


@pytest.mark.parametrize("window", [20, 60, 61, 1 << 30, 2147483647])
def test_windows_about_and_past_the_length(window):
    rng = np.random.default_rng(30)
    Batch(rng, [(59, 1), (-2, 4), (20, 40)], 4, 2, 64, 16, "f16").device(window=window).run().check()


@pytest.mark.parametrize("act,D", [("bf16", 128), ("f16", 64)])
def test_enough_units_for_whole_ones(act, D):
    """So many tiles of rows that every workgroup takes one, some workgroups more than the batch has."""
    rng = np.random.default_rng(31)
    # tiles of 128 rows: 4 of 24 heads in five requests, 35 of 32 heads in one
    Batch(rng, [(0, 150), (10, 1), (30, 90), (0, 0), (0, 40)] * 12, 24, 24, D, 32, act).device().run().check()
    Batch(rng, [(0, 4400)], 32, 32, D, 64, act).device().run().check()


@pytest.mark.parametrize("act,heads,kv,D,B", [("f16", 8, 2, 128, 64), ("bf16", 4, 4, 64, 16), ("bf16", 28, 4, 128, 32)])
@pytest.mark.parametrize("requests,window", [([(3000, 64)], 0), ([(0, 700), (2500, 20), (1200, 90), (700, 1)], 0), ([(2500, 150), (100, 9)], 1200),
                                             ([(0, 900), (1500, 33)], 600)])
def test_pieces_on_long_contexts_are_cut_and_joined(act, heads, kv, D, B, requests, window):
    """Tiles of many rows in shares of several steps, tiles and requests partly filled."""
    rng = np.random.default_rng(33)
    b = Batch(rng, requests, heads, kv, D, B, act, pad_o=8).device(window=window)
    first = b.run().check()
    for _ in range(3):
        b.dout.fill_(float("nan"))
        assert np.array_equal(b.run().output(), first)


@pytest.mark.parametrize("D", [64, 128])
def test_numbers_that_are_none_in_one_share(D):
    """A value that is none, in the middle of a long context: its dim of the rows that see it, in whatever share it lies."""
    rng = np.random.default_rng(34)
    cached, fresh = 1800, 200
    b = Batch(rng, [(cached, fresh)], 4, 2, D, 32, "bf16")
    at = cached + 77
    slot = int(b.table[0, at // 32]) * 32 + at % 32
    b.cache.codes[1][slot // 32, 1, slot % 32, 5] = K.NAN_CODE
    want_nan = np.zeros((fresh, 4, D), bool)
    want_nan[77:, 2:, 5] = True
    b.device().run()
    got = b.output()
    assert np.array_equal(np.isnan(got), want_nan)
    b.cache.codes[1][b.cache.codes[1] == K.NAN_CODE] = 0
    out, bound = b.reference()
    sees = np.zeros_like(want_nan)
    sees[77:, 2:] = True                                            # (those also lose the value's weight)
    assert (np.abs(got - out)[~sees] <= bound[~sees]).all()


@pytest.mark.parametrize("act,D", [("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("window", [0, 500])
def test_more_requests_than_lanes_some_of_them_cut(act, D, window):
    """More than 64 requests: long ones in parts between short ones, of few rows and of many."""
    rng = np.random.default_rng(35)
    kinds = [(20, 1), (4000, 1), (0, 0), (90, 30), (1700, 40), (300, 5), (5, 0), (0, 150), (33, 1), (2000, 2)]
    b = Batch(rng, [kinds[i % 10] if i % 30 < 11 else (int(rng.integers(0, 200)), 1) for i in range(150)], 8, 2, D, 32, act)
    first = b.device(window=window).run().check()
    b.dout.fill_(float("nan"))
    assert np.array_equal(b.run().output(), first)
    ones = Batch(rng, [(4000, 1) if i == 70 else (i, 1) for i in range(90)], 4, 1, D, 32, act).device(window=window)
    ones.run().check()


def test_mixed_batches_of_heads_alone():
    rng = np.random.default_rng(32)
    Batch(rng, [(900, 1), (0, 300), (3, 1), (500, 17), (64, 16)], 3, 3, 128, 16, "f16").device().run().check()


def test_bounds_larger_than_needed_change_nothing():
    rng = np.random.default_rng(28)
    b = Batch(rng, [(600, 1), (33, 1)], 8, 2, 128, 32, "f16").device()
    want = b.run().check()
    b.device(max_length=40000)
    assert np.array_equal(b.run().output(), want)


def test_offsets_past_32_bits():
    """Pages behind the first 4 GiB of codes."""
    B, kv, D = 128, 8, 128
    n = (5 << 30) // (B * kv * D)
    codes = [torch.empty(n * kv * B * D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty(n * kv, dtype=torch.uint8, device="cuda") for _ in range(2)]
    rng = np.random.default_rng(29)
    blocks = [n - 1, n - 7, n // 2 + 1]
    small = K.Cache(3, B, kv, D)
    rows = rows_of(rng, 300, kv, D, "f16")
    at = np.arange(300)
    small.append(rows, at)
    desc = G.make_kv_cache(codes[0].data_ptr(), codes[1].data_ptr(), scales[0].data_ptr(), scales[1].data_ptr(), n, B, kv, D)
    slots = i32(np.array(blocks)[at // B] * B + at % B)
    dev = [torch.from_numpy(x.reshape(300, -1)).half().cuda() for x in rows]
    G.glowq_kv_append(desc, dev[0].data_ptr(), kv * D, dev[1].data_ptr(), kv * D, G.GLOWQ_F16, slots.data_ptr(), 300, stream())
    back = [torch.empty_like(x) for x in dev]
    G.glowq_kv_gather(desc, slots.data_ptr(), 300, back[0].data_ptr(), kv * D, back[1].data_ptr(), kv * D, G.GLOWQ_F16, stream())
    torch.cuda.synchronize()
    for w in range(2):
        assert np.array_equal(back[w].double().cpu().numpy().reshape(300, kv, D), small.tokens(w, at))
    b = Batch(rng, [(299, 1)], 16, kv, D, B, "f16", spare=0)
    b.cache, b.table = small, np.array([[0, 1, 2]])
    b.used = list(range(300))
    b.device()
    want = b.run().check()
    b.dc.desc = desc
    b.dtable.copy_(i32([blocks]))
    b.dout.fill_(float("nan"))
    assert np.array_equal(b.run().output(), want)
