"""GPU parity of the latent operators with their oracle: the cache's bytes equal, per-head maps and both forms of attention within the
bounds that their roundings allow (tests/latent_util.py derives them)."""
import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from oracle import latent_oracle as L
from gpu_util import ACT_CODE, TORCH_ACT, stream
from kv_util import act_round, i32
from latent_util import ROUNDOFF, TINY, Absorbed, DeviceLatents, Expanded, Rope, Rows, random_latents, rope_rows, within

pytestmark = pytest.mark.gpu
ACTS = pytest.mark.parametrize("act", ["f16", "bf16"])


# ---- the cache ------------------------------------------------------------------------------
@ACTS
@pytest.mark.parametrize("latent,rope,T,B,r", [(512, 64, 1, 16, 64), (512, 32, 67, 128, 0), (256, 64, 300, 32, 32), (256, 32, 5, 64, 32)])
def test_tokens_into_the_cache_and_back(act, latent, rope, T, B, r):
    rng = np.random.default_rng(T)
    n = T // B + 4
    d = DeviceLatents(random_latents(rng, n, B, latent, rope, act), used=[])
    slots = rng.permutation(n * B)[:T]
    if T > 3:
        slots[:2] = (-1, n * B)
    # magnitudes from far below the smallest grid to the type's largest, tokens of zeros, numbers that are none
    size = np.exp2(rng.uniform(-24, 15.9 if act == "f16" else 60, T))
    c, kr = rng.uniform(-1, 1, (T, latent)) * size[:, None], rng.standard_normal((T, 1, rope))
    if T > 10:
        c[3], c[4, 7], c[5, 9], c[6, :] = 0.0, np.inf, np.nan, np.nan
        c[7], c[8, 5] = 65504.0, 65504.0
        kr[9, 0, 1] = np.inf
    c, kr = act_round(c, act), act_round(kr, act)
    positions = rng.integers(0, 100000, T)
    positions[T // 2] = -3
    q, rp = act_round(rng.standard_normal((T, 5, rope)), act), Rope(r, "pairs", "ramp") if r else None
    x, dq, dout = Rows(np.concatenate([c, kr[:, 0]], 1)[:, None], act, 0, 8), Rows(q, act, 16, 0), Rows(np.zeros_like(q), act, 8, 8, filled=False)
    row, dslots, dpositions = x.buf.data_ptr(), i32(slots), i32(positions)
    G.glowq_latent_append(d.desc, rp and rp.desc, rope_rows(dq, dout) if r else None, row, x.ld, row + 2 * latent, x.ld, dslots.data_ptr(),
                          dpositions.data_ptr() if r else 0, T, stream())
    torch.cuda.synchronize()
    d.o.append(c, kr[:, 0], slots)
    at = slots[(slots >= 0) & (slots < n * B)]
    assert np.array_equal(d.scales.cpu().numpy()[at], (d.o.exps[at] + 127).astype(np.uint8))
    codes = d.codes.cpu().numpy()
    assert np.array_equal(K.VALUES[codes[at]], K.VALUES[d.o.codes[at]], equal_nan=True)
    rest = np.setdiff1d(np.arange(n * B), at)
    assert (codes[rest] == 0xFF).all() and np.isnan(d.ropes.float().cpu().numpy()[rest]).all()
    # read back: the same numbers; zeros where there is no slot
    oc, orr = Rows(np.zeros((T, 1, latent)), act, 0, 8, filled=False), Rows(np.zeros((T, 1, rope)), act, 0, 16, filled=False)
    G.glowq_latent_gather(d.desc, dslots.data_ptr(), T, oc.buf.data_ptr(), oc.ld, orr.buf.data_ptr(), orr.ld, stream())
    want = d.o.latents(slots)
    assert np.array_equal(oc.numbers()[:, 0], want, equal_nan=True)
    got, live = orr.numbers()[:, 0], np.isin(slots, at)
    assert not got[~live].any()
    if not r:
        assert np.array_equal(got[live], kr[live, 0], equal_nan=True)
        return
    turned = rp.rotate(kr, np.maximum(positions, 0))
    fine = live & np.isfinite(kr).all((1, 2))
    assert (np.abs(got - turned[:, 0])[fine] <= (rp.slack(kr) + ROUNDOFF[act] * np.abs(turned) + TINY[act])[fine, 0]).all()
    rows = dout.numbers()
    assert np.isnan(rows[positions < 0]).all()
    turned = rp.rotate(q, positions)
    bound = rp.slack(q) + ROUNDOFF[act] * np.abs(turned) + TINY[act]
    assert (np.abs(rows - turned) <= bound)[positions >= 0].all()


def test_offsets_beyond_32_bits():
    # the last blocks of a cache of 5 GB
    B, latent, rope, n = 128, 512, 64, 75000
    codes, scales = torch.full((n * B, latent), 0xFF, dtype=torch.uint8, device="cuda"), torch.full((n * B,), 255, dtype=torch.uint8, device="cuda")
    ropes = torch.full((n * B, rope), float("nan"), dtype=torch.bfloat16, device="cuda")
    desc = G.make_latent_cache(codes=codes.data_ptr(), scales=scales.data_ptr(), ropes=ropes.data_ptr(), n_blocks=n, block_tokens=B, latent_dim=latent,
                               rope_dim=rope, act_dtype=G.GLOWQ_BF16)
    rng = np.random.default_rng(1)
    b = Absorbed(rng, [(150, 1)], 16, latent, rope, B, "bf16", spare=0)
    order = np.array([n - 1, n - 3])
    slots = order[np.arange(151) // B] * B + np.arange(151) % B
    c = b.cache.latents(L.slots_of(b.table, 0, 151, B, 2))
    kr = b.cache.key_parts(L.slots_of(b.table, 0, 151, B, 2))
    dc, dr, dslots = Rows(c[:, None], "bf16"), Rows(kr[:, None], "bf16"), i32(slots)
    G.glowq_latent_append(desc, None, None, dc.buf.data_ptr(), dc.ld, dr.buf.data_ptr(), dr.ld, dslots.data_ptr(), 0, 151, stream())
    b.device()
    b.dtable = i32(order[None])
    b.desc.table, b.dc.desc = b.dtable.data_ptr(), desc
    b.run().check()


# ---- per-head maps ----------------------------------------------------------------------------
@ACTS
@pytest.mark.parametrize("T,heads,d_in,d_out,gap", [(1, 1, 32, 16, 0), (16, 3, 128, 512, 64), (17, 5, 512, 128, 0), (33, 2, 64, 256, 8), (65, 4, 256, 64, 0),
                                                    (200, 7, 160, 48, 16), (5, 2, 800, 32, 8), (20, 2, 608, 16, 8), (40, 3, 672, 16, 0)])
def test_head_maps(act, T, heads, d_in, d_out, gap):
    rng = np.random.default_rng(T)
    x, w = act_round(rng.standard_normal((T, heads, d_in)), act), act_round(rng.standard_normal((heads, d_out, d_in)), act)
    dx, dy, dw = Rows(x, act, gap, 8), Rows(np.zeros((T, heads, d_out)), act, gap, 16, filled=False), Rows(w, act)
    G.glowq_head_maps(dx.buf.data_ptr(), dx.ld, dx.lh, dw.buf.data_ptr(), dy.buf.data_ptr(), dy.ld, dy.lh, heads, d_in, d_out, ACT_CODE[act], T, stream())
    want = np.einsum("thi,hoi->tho", x, w)
    size = np.einsum("thi,hoi->tho", np.abs(x), np.abs(w))
    within(dy.numbers(), want, ROUNDOFF[act] * np.abs(want) + (d_in + 4) * 2.0 ** -24 * size + TINY[act])


# ---- absorbed attention --------------------------------------------------------------------
@ACTS
@pytest.mark.parametrize("heads,latent,rope,B", [(1, 512, 64, 16), (16, 512, 32, 64), (20, 256, 64, 32), (40, 256, 32, 128), (128, 512, 64, 64)])
def test_absorbed_single_tokens(act, heads, latent, rope, B):
    rng = np.random.default_rng(heads)
    # one token in all, around the tiles' and the blocks' borders, long ones, none
    lengths = [1, 2, 15, 63, 64, 65, 127, 128, 129, 500, 1500]
    b = Absorbed(rng, [(n - 1, 1) for n in lengths] + [(30, 0)], heads, latent, rope, B, act, pad_q=8, pad_o=16)
    b.device().run().check()


@ACTS
@pytest.mark.parametrize("heads,latent,rope,B", [(3, 256, 32, 16), (16, 512, 64, 64), (7, 512, 32, 32), (64, 256, 64, 128)])
def test_absorbed_pieces(act, heads, latent, rope, B):
    rng = np.random.default_rng(heads + 1)
    b = Absorbed(rng, [(0, 1), (0, 5), (60, 9), (0, 64), (130, 1), (1000, 31), (63, 2), (5, 0)], heads, latent, rope, B, act)
    b.device(max_fresh=70, max_length=3000).run().check()


@pytest.mark.parametrize("n,heads,cached", [(1, 128, 20000), (2, 16, 9000), (70, 16, 300), (300, 5, 40)])
def test_absorbed_long_and_many(n, heads, cached):
    rng = np.random.default_rng(n)
    b = Absorbed(rng, [(int(rng.integers(0, cached) if n > 2 else cached - 7 * i), 1) for i in range(n)], heads, 512, 64, 64, "bf16")
    first = b.device().run().check()
    assert np.array_equal(first, b.run().output())               # the same call gives the same bits


def test_absorbed_beyond_the_callers_bounds():
    rng = np.random.default_rng(6)
    b = Absorbed(rng, [(100, 5), (20, 2)], 16, 256, 32, 32, "f16")
    b.device(max_fresh=2, max_length=64).run()
    out = b.output()
    # rows past max_fresh stay unwritten, keys past max_length are left out, the others keep their positions
    assert np.isnan(out[2:5]).all()
    n = [min(v, 64) for v in b.lengths]
    want = L.absorbed(b.cache, b.q[:2], b.table[:1], [102], [0, 2], b.scale)
    slots = L.slots_of(b.table, 0, 64, 32, b.cache.n_blocks)
    lat = b.cache.latents(slots)
    k = np.concatenate([lat, b.cache.key_parts(slots)], 1)
    for i in range(2):
        for h in range(16):
            s = np.exp(k @ b.q[i, h] * b.scale)
            assert np.allclose(out[i, h], s @ lat / s.sum(), rtol=0, atol=4e-3)
    assert np.allclose(out[5:7], L.absorbed(b.cache, b.q[5:7], b.table[1:], [22], [0, 2], b.scale), rtol=0, atol=4e-3) and want.shape and n


@ACTS
def test_absorbed_scales_far_apart(act):
    # tokens whose scales differ by up to 2^20 (2^40), tokens of zeros with the largest weights
    rng = np.random.default_rng(7)
    b = Absorbed(rng, [(400, 3), (37, 1)], 20, 256, 32, 16, act, q_scale=0.05)
    b.cache.exps[:] = rng.integers(-15 if act == "f16" else -34, 6, b.cache.exps.shape)
    b.cache.codes[::5], b.cache.exps[::5] = 0, -15 if act == "f16" else -64
    b.scale = 1.0 / 64
    b.device().run().check()


def test_absorbed_at_the_upper_end_of_bfloat16():
    # latents up to 2^127, queries as much smaller: sums of weights relative to the largest value are about 2^-118
    rng = np.random.default_rng(18)
    b = Absorbed(rng, [(700, 3), (70, 1)], 20, 256, 32, 16, "bf16")
    b.cache.exps[:] = rng.integers(112, 119, b.cache.exps.shape)
    b.q[..., :256] *= 2.0 ** -118
    b.q[np.abs(b.q) < 2.0 ** -126] = 0                              # (no subnormal numbers)
    b.scale = 1.0 / 128
    b.device().run().check()


@ACTS
def test_absorbed_scores_far_apart(act):
    rng = np.random.default_rng(8)
    b = Absorbed(rng, [(700, 2), (64, 1)], 16, 512, 64, 64, act, q_scale=30.0)
    b.device().run().check()


@ACTS
@pytest.mark.parametrize("latent", [256, 512])
def test_absorbed_rows_that_see_no_key_and_blocks_outside(act, latent):
    rng = np.random.default_rng(9)
    b = Absorbed(rng, [(100, 4), (0, 3), (200, 1), (64, 1)], 10, latent, 32, 32, act)
    b.table[0, 1], b.table[0, 3] = -1, b.cache.n_blocks           # pieces of it are gone
    b.table[2, :] = -7                                             # all of it
    b.lengths[1] = 1                                               # three new tokens of one in all: two come before the first
    out = b.device().run().check()
    assert not out[4:6].any() and out[6].any() and not out[7].any()


@ACTS
@pytest.mark.parametrize("heads,latent", [(5, 512), (40, 256)])
def test_absorbed_hidden_nan_stays_hidden(act, heads, latent):
    rng = np.random.default_rng(10)
    b = Absorbed(rng, [(90, 8), (10, 3)], heads, latent, 32, 32, act)
    slots = L.slots_of(b.table, 0, 98, 32, b.cache.n_blocks)
    clean = b.device().run().check().copy()
    b.cache.codes[slots[94], 17] = 0x7F                            # token 4 of the new ones
    b.cache.ropes[slots[96], 3] = np.inf                           # token 6
    out = b.device().run().output()
    assert np.array_equal(out[:4], clean[:4]) and np.array_equal(out[8:], clean[8:])
    assert np.isnan(out[4:8]).all()


@pytest.mark.parametrize("heads,latent,act", [(3, 512, "bf16"), (40, 256, "f16")])
def test_absorbed_parts_of_hundreds_of_steps(heads, latent, act):
    # more units than the machine holds, so that parts are long and blocks are looked up again and again; all requests read
    # the same blocks
    rng, n = np.random.default_rng(19), 300
    b = Absorbed(rng, [(20000, 1)], heads, latent, 32, 128, act, q_scale=0.2)
    b.fresh, b.lengths = [1] * n, [int(v) for v in rng.integers(17000, 20002, n)]
    b.starts, b.T = np.arange(n + 1), n + 1
    b.table = np.repeat(b.table, n, 0)
    b.q = act_round(rng.standard_normal((b.T, heads, latent + 32)) * 0.2, act)
    out = b.device().run().output()
    b.fresh = [int(r % 25 == 0) for r in range(n)]                  # the reference takes its time
    want, bound = b.reference()
    within(out[::25], want[::25], bound[::25])
    assert np.isfinite(out).all()


def test_absorbed_on_two_streams_at_once():
    rng = np.random.default_rng(20)
    calls = [Absorbed(rng, [(3000 + 100 * i, 1), (50, 2)], 64, 512, 64, 64, "bf16").device() for i in range(2)]
    alone = [b.run().check() for b in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, s in zip(calls, streams):
            with torch.cuda.stream(s):
                b.run()
    torch.cuda.synchronize()
    assert all(np.array_equal(b.output(), want) for b, want in zip(calls, alone))


def test_absorbed_in_a_graph_on_its_stream_with_a_shared_workspace():
    rng = np.random.default_rng(11)
    b, c = (Absorbed(rng, [(900, 1), (64, 1)], 16, 512, 64, 64, "bf16") for _ in range(2))
    b.device(), c.device()
    ws = torch.full((max(b.ws.numel(), c.ws.numel()),), 0xFF, dtype=torch.uint8, device="cuda")
    b.ws = c.ws = ws
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for x in (b, c):
        with torch.cuda.stream(side):
            x.run()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                x.run()
            graphs.append(g)
    for n in range(3):
        for x in (b, c):
            x.dout.view[:] = float("nan")
            x.dlengths.copy_(i32([901 - 300 * n, 65 - n]))
            x.lengths = [901 - 300 * n, 65 - n]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        b.check(), c.check()


# ---- expanded attention -------------------------------------------------------------------
@ACTS
@pytest.mark.parametrize("heads,nope,rope,beside", [(1, 128, 64, True), (3, 64, 32, False), (2, 128, 32, True), (5, 64, 64, True)])
def test_expanded_prompts_and_pieces(act, heads, nope, rope, beside):
    rng = np.random.default_rng(heads)
    b = Expanded(rng, [(0, 1), (0, 2), (0, 63), (0, 64), (0, 65), (0, 129), (0, 300), (200, 1), (64, 64), (1000, 33), (30, 0), (77, 130)], heads, nope, rope, act,
                 pad=8 * heads, gap=8 * (heads - 1), beside=beside)
    b.device().run().check()


@pytest.mark.parametrize("requests,heads", [([(0, 1500)], 2), ([(9000, 40)], 3), ([(4000, 200), (0, 700), (6000, 1)], 2), ([(0, 3)] * 90, 2)])
def test_expanded_long_and_many(requests, heads):
    rng = np.random.default_rng(heads)
    b = Expanded(rng, requests, heads, 128, 64, "bf16")
    first = b.device().run().check()
    assert np.array_equal(first, b.run().output())


@ACTS
def test_expanded_scores_far_apart_and_rows_that_see_no_key(act):
    rng = np.random.default_rng(2)
    b = Expanded(rng, [(0, 200), (300, 20), (0, 5)], 2, 64, 32, act, q_scale=20.0)
    b.lengths[2] = 2                                               # five new tokens of two in all: three come before the first
    out = b.device().run().check()
    assert not out[220:223].any() and out[223:].any()


@ACTS
@pytest.mark.parametrize("nope,rope", [(64, 32), (128, 64)])
def test_expanded_hidden_nan_stays_hidden(act, nope, rope):
    rng = np.random.default_rng(3)
    b = Expanded(rng, [(70, 60), (0, 40)], 2, nope, rope, act)
    clean = b.device().run().check().copy()
    k0, k1 = b.key_starts
    b.v[k0 + 100, 0, 5], b.k[k0 + 110, 1, 3], b.kr[k1 + 30, 2], b.v[k1 + 20, 1, 9] = np.nan, np.nan, np.inf, -np.inf
    out = b.device().run().output()
    same = np.ones(out.shape, bool)
    same[30:60, 0, 5] = False                                      # a value: its dim, in rows that see it
    same[40:60, 1] = False                                         # a key: everything
    same[90:, :] = False                                           # ... of both heads
    same[80:, 1, 9] = False
    assert np.array_equal(out[same], clean[same])
    assert np.isnan(out[30:60, 0, 5]).all() and np.isnan(out[40:60, 1]).all() and not np.isfinite(out[80:, 1, 9]).any()


def test_expanded_in_a_graph():
    rng = np.random.default_rng(4)
    b = Expanded(rng, [(3000, 100), (0, 50)], 2, 128, 64, "bf16").device()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            b.run()
    for n in range(3):
        b.dout.view[:] = float("nan")
        b.lengths = [3100 - 700 * n, 50]
        b.dlengths.copy_(i32(b.lengths))
        torch.cuda.synchronize()
        g.replay()
        b.check()


# ---- a step as a program makes it ------------------------------------------------------------
@ACTS
def test_tokens_in_pieces_agree_with_their_prompt(act):
    """The same tokens through the cache, absorbed, piece by piece, and as one expanded prompt from what the cache holds."""
    rng = np.random.default_rng(12)
    heads, N, latent, rope, n, B = 6, 64, 256, 32, 150, 32
    rp, blocks = Rope(rope, "pairs", "ramp"), 8
    u = ROUNDOFF[act]
    c, kr, q = (act_round(rng.standard_normal(s), act) for s in ((n, latent), (n, 1, rope), (n, heads, N + rope)))
    up, down = (act_round(rng.standard_normal((heads, N, latent)) / 16, act) for _ in range(2))
    d = DeviceLatents(L.LatentCache(blocks, B, latent, rope, act))
    table = i32(rng.permutation(blocks)[None])
    out, step = torch.empty(n, heads, N, dtype=TORCH_ACT[act], device="cuda"), i32([0])
    dup_t = torch.from_numpy(up).to(TORCH_ACT[act]).cuda().transpose(1, 2).contiguous()       # queries into the latents: [head][latent][N]
    ddown = torch.from_numpy(down).to(TORCH_ACT[act]).cuda()
    at, code = 0, ACT_CODE[act]
    for f in (100, 1, 1, 17, 1, 30):
        dx, dq = Rows(np.concatenate([c, kr[:, 0]], 1)[at:at + f, None], act), Rows(q[at:at + f], act)
        qa, oa, o = (Rows(np.zeros((f, heads, w)), act, filled=False) for w in (latent + rope, latent, N))
        cached, fresh, starts, lengths = i32([at]), i32([f]), i32([0, 0]), i32([0])
        slots, positions, taken = i32([0] * f), i32([0] * f), i32([0])
        free = i32(np.arange(1))
        G.glowq_kv_plan(G.make_kv_step(cached=cached.data_ptr(), fresh=fresh.data_ptr(), free_blocks=table.data_ptr() + 4 * (-(-at // B)), table=table.data_ptr(),
                                       lengths=lengths.data_ptr(), starts=starts.data_ptr(), slots=slots.data_ptr(), positions=positions.data_ptr(),
                                       taken=taken.data_ptr(), n_requests=1, n_free=blocks - -(-at // B), table_width=blocks, max_tokens=f, block_tokens=B), stream())
        G.glowq_head_maps(dq.buf.data_ptr(), dq.ld, dq.lh, dup_t.data_ptr(), qa.buf.data_ptr(), qa.ld, qa.lh, heads, N, latent, code, f, stream())
        G.glowq_latent_append(d.desc, rp.desc, rope_rows(dq, qa, at_x=N, at_y=latent), dx.buf.data_ptr(), dx.ld, dx.buf.data_ptr() + 2 * latent, dx.ld,
                              slots.data_ptr(), positions.data_ptr(), f, stream())
        att = G.make_latent_attention(q=qa.buf.data_ptr(), out=oa.buf.data_ptr(), table=table.data_ptr(), lengths=lengths.data_ptr(), starts=starts.data_ptr(),
                                      ldq=qa.ld, ldo=oa.ld, table_width=blocks, n_requests=1, T=f, heads=heads, max_fresh=f, max_length=n, scale=0.1)
        ws = torch.empty(G.glowq_latent_attention_workspace_bytes(d.desc, att), dtype=torch.uint8, device="cuda")
        G.glowq_latent_attention(d.desc, att, ws.data_ptr(), ws.numel(), stream())
        G.glowq_head_maps(oa.buf.data_ptr(), oa.ld, oa.lh, ddown.data_ptr(), o.buf.data_ptr(), o.ld, o.lh, heads, latent, N, code, f, stream())
        torch.cuda.synchronize()
        assert int(lengths[0]) == at + f and free.numel()
        out[at:at + f] = o.view
        at += f
    # expanded: latents read back, keys and values of them, the rotated key parts, the rotated queries
    all_slots = (table[0].long()[torch.arange(n, device="cuda") // B] * B + torch.arange(n, device="cuda") % B).int()
    lat, parts = Rows(np.zeros((n, 1, latent)), act, filled=False), Rows(np.zeros((n, 1, rope)), act, filled=False)
    G.glowq_latent_gather(d.desc, all_slots.data_ptr(), n, lat.buf.data_ptr(), lat.ld, parts.buf.data_ptr(), parts.ld, stream())
    x = lat.numbers()[:, 0]
    k, v = (act_round(np.einsum("jl,hnl->jhn", x, w), act) for w in (up, down))
    dk, dv, dq, oe = Rows(k, act), Rows(v, act), Rows(q, act), Rows(np.zeros((n, heads, N)), act, filled=False)
    order = i32(np.arange(n))
    G.glowq_rotate(rp.desc, [rope_rows(dq, dq, at_x=N, at_y=N)], rope, code, order.data_ptr(), n, stream())
    zero, total = i32([0]), i32([n])
    rows = i32([0, n])
    e = G.make_expanded_attention(q=dq.buf.data_ptr(), k=dk.buf.data_ptr(), k_rope=parts.buf.data_ptr(), v=dv.buf.data_ptr(), out=oe.buf.data_ptr(),
                                  starts=rows.data_ptr(), key_starts=zero.data_ptr(), lengths=total.data_ptr(), ldq=dq.ld, lhq=dq.lh, ldk=dk.ld, lhk=dk.lh,
                                  ldr=parts.ld, ldv=dv.ld, lhv=dv.lh, ldo=oe.ld, n_requests=1, T=n, keys=n, heads=heads, nope_dim=N, rope_dim=rope, v_dim=N,
                                  act_dtype=code, max_fresh=n, max_length=n, scale=0.1)
    ws = torch.empty(G.glowq_expanded_attention_workspace_bytes(e), dtype=torch.uint8, device="cuda")
    G.glowq_expanded_attention(e, ws.data_ptr(), ws.numel(), stream())
    a, b = out.double().cpu().numpy(), oe.numbers()
    # between the two: q', keys, values, weights, o and the results are rounded, each u of what it is; rounded scores move weights by
    # u sum |q k| scale, in the sum and in the parts
    qr = rp.rotate(np.concatenate([q[..., N:], q[..., :N]], -1), np.arange(n))
    qn, qp, pr = q[..., :N], qr[..., :rope], parts.numbers()[:, 0]
    with np.errstate(all="ignore"):
        for t in (0, 50, 99, 101, 149):
            for h in range(heads):
                s = (x[:t + 1] @ up[h].T @ qn[t, h] + pr[:t + 1] @ qp[t, h]) * 0.1
                size = ((np.abs(x[:t + 1]) @ np.abs(up[h]).T @ np.abs(qn[t, h])) + np.abs(pr[:t + 1]) @ np.abs(qp[t, h])) * 0.1
                w = np.exp(s - s.max())
                w /= w.sum()
                mag = w @ (np.abs(x[:t + 1]) @ np.abs(down[h]).T)
                bound = mag * u * (6 + 4 * size.max()) + 1e-6
                want = w @ (x[:t + 1] @ down[h].T)
                assert (np.abs(a[t, h] - want) <= bound).all() and (np.abs(b[t, h] - want) <= bound).all(), (t, h)
