"""Glue for the tests of rotary positions and latent attention: descriptors from seeds, the calls of the C ABI through the
binding, references in 64 bits with bounds of what the kernels' roundings allow."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from oracle import latent_oracle as L
from oracle import rope_oracle as R
from gpu_util import ACT_CODE, TORCH_ACT, stream
from kv_util import act_round, i32
from test_oracle_latent import spec

# half a step of the type, relative, and its smallest step's half
ROUNDOFF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}
# An error of a rotated number in fp32, of |a| + |b|: the angle's fraction (its conversion, two products) 2.4, the series 2, the
# magnitude 1, products and sum 3, with what they multiply: below 12 times 2^-24
TURN = 12 * 2.0 ** -24


def on_gpu(x, act):
    return torch.from_numpy(np.ascontiguousarray(x)).to(TORCH_ACT[act]).cuda()


class Rope:
    def __init__(self, rotary_dim, layout="halves", scaling="plain"):
        self.r, self.layout = rotary_dim, layout
        self.turns, self.magnitude = G.glowq_rope_turns(spec(rotary_dim, scaling))
        self.dev = torch.tensor([t - (1 << 64) if t >> 63 else t for t in self.turns], dtype=torch.int64, device="cuda")
        self.desc = G.make_rope(turns=self.dev.data_ptr(), rotary_dim=rotary_dim,
                                layout=G.GLOWQ_ROPE_HALVES if layout == "halves" else G.GLOWQ_ROPE_PAIRS, magnitude=self.magnitude)

    def rotate(self, x, positions):
        return R.rotate(x, self.turns, positions, self.layout, self.magnitude)

    def slack(self, x):
        """The bound of the error before the last rounding."""
        return TURN * R.reach(np.abs(x), self.r, self.layout, self.magnitude)


class Rows:
    """A tensor of heads in memory with gaps: NaN between heads, right of the rows and behind them, which no call may touch."""

    def __init__(self, x, act, gap=0, pad=0, filled=True):
        T, h, d = x.shape
        self.T, self.h, self.d, self.lh, self.ld = T, h, d, d + gap, h * (d + gap) + pad
        self.buf = torch.full((T + 2, self.ld), float("nan"), dtype=TORCH_ACT[act], device="cuda")
        if filled:
            self.view[:] = torch.from_numpy(x).to(TORCH_ACT[act]).cuda()

    @property
    def view(self):
        return self.buf[:self.T, :self.h * self.lh].view(self.T, self.h, self.lh)[:, :, :self.d]

    def numbers(self):
        torch.cuda.synchronize()
        keep = self.view.clone()
        self.view[:] = float("nan")
        assert torch.isnan(self.buf).all(), "written beside the rows"
        self.view[:] = keep
        return keep.double().cpu().numpy()


def rope_rows(x: Rows, y: Rows, at_x=0, at_y=0, heads=None):
    size = x.buf.element_size()
    return G.make_rope_rows(x=x.buf.data_ptr() + at_x * size, y=y.buf.data_ptr() + at_y * size, heads=heads or x.h, ldx=x.ld, lhx=x.lh, ldy=y.ld, lhy=y.lh)


class DeviceLatents:
    """The bytes of an oracle cache on the GPU; what no request uses is NaN, scales of such tokens 255."""

    def __init__(self, cache: L.LatentCache, used=None):
        self.o = cache
        codes, scales, ropes = cache.codes.copy(), (cache.exps + 127).astype(np.uint8), cache.ropes.copy()
        if used is not None:
            free = np.setdiff1d(np.arange(len(scales)), np.asarray(used, np.int64))
            codes[free], scales[free], ropes[free] = 0xFF, 255, np.nan
        self.codes, self.scales, self.ropes = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), on_gpu(ropes, cache.act)
        self.desc = G.make_latent_cache(codes=self.codes.data_ptr(), scales=self.scales.data_ptr(), ropes=self.ropes.data_ptr(), n_blocks=cache.n_blocks,
                                        block_tokens=cache.B, latent_dim=cache.latent, rope_dim=cache.rope, act_dtype=ACT_CODE[cache.act])


def random_latents(rng, n_blocks, B, latent, rope, act, spread=1):
    c = L.LatentCache(n_blocks, B, latent, rope, act)
    c.codes[:] = K.encode(np.clip(rng.standard_normal(c.codes.shape) * 72.0, -448, 448))
    c.exps[:] = rng.integers(-6 - spread, -5 + spread, c.exps.shape)
    c.ropes[:] = act_round(rng.standard_normal(c.ropes.shape), act)
    return c


def tables(rng, requests, B, spare):
    """(table, blocks in all, slots in use)"""
    n = [max(0, -(-(c + f) // B)) for c, f in requests]
    ids = rng.permutation(sum(n) + spare)
    table, at = np.full((len(requests), max(1, max(n))), -1, np.int64), 0
    for r, k in enumerate(n):
        table[r, :k] = ids[at:at + k]
        at += k
    used = [int(table[r, j // B]) * B + j % B for r, (c, f) in enumerate(requests) for j in range(max(c + f, 0))]
    return table, sum(n) + spare, used


def softmax_reference(q, k, v, see, scale, act, dims, v_exp=None):
    """(out, bound) of one head's rows over its keys, all in float64 on the GPU.  The bound on |error|: weights and the result rounded to
    the type, u each of sum p |v| and |out| (twice where l is the sum of the rounded weights: counted always); scores in fp32, their sums off by
    (dims + 4) 2^-24 sum |q k| scale at most, in the weights and in their sum; sums over L keys; the exponential's last
    places; weights below the normal range of binary16, each off by 2^-25 in units of at most the largest weight, times 448 of its grid."""
    u, n = ROUNDOFF[act], k.shape[0]
    if n == 0:
        zero = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64, device="cuda")
        return zero, zero + 2.0 ** -24
    s = (q @ k.t().contiguous() * scale).masked_fill(~see, -math.inf)
    w = torch.softmax(s, 1)
    w[~see.any(1)] = 0.0
    size = (q.abs() @ k.abs().t().contiguous() * scale).masked_fill(~see, 0.0).amax(1, keepdim=True)
    out, mag = w @ v, w @ v.abs()
    eps = 2.0 ** -24 * (2 * (dims + 4) * size + 2 * n + 64)
    small = 0.0
    if act == "f16":
        if v_exp is None:
            small = n * 2.0 ** -25 * (v.abs().amax(1)[None] * see).amax(1, keepdim=True)
        else:
            # the token with the largest s + e has a weight of one at least
            at = (s / math.log(2.0) + v_exp[None]).masked_fill(~see, -math.inf).argmax(1)
            small = n * 2.0 ** -25 * 448 * torch.exp2(v_exp[at])[:, None]
    return out, (2 * u + eps) * mag + u * out.abs() + small + TINY[act] + 2.0 ** -60


class Absorbed:
    """Requests (cached, fresh) over a random latent cache; the fresh tokens are in it already."""

    def __init__(self, rng, requests, heads, latent, rope, B, act, spare=3, q_scale=0.5, pad_q=0, pad_o=0, extra_rows=2, spread=1):
        self.act, self.heads, self.latent, self.rope, self.B = act, heads, latent, rope, B
        self.fresh, self.lengths = [f for _, f in requests], [c + f for c, f in requests]
        self.starts = np.concatenate([[0], np.cumsum(self.fresh)]).astype(int)
        self.table, blocks, self.used = tables(rng, requests, B, spare)
        self.cache = random_latents(rng, blocks, B, latent, rope, act, spread)
        self.T = max(1, int(self.starts[-1])) + extra_rows
        self.q = act_round(rng.standard_normal((self.T, heads, latent + rope)) * q_scale, act)
        self.pad_q, self.pad_o, self.scale = pad_q, pad_o, 1.0 / math.sqrt(latent // 4 + rope)

    def device(self, max_fresh=None, max_length=None):
        self.dc = DeviceLatents(self.cache, self.used)
        self.dq, self.dout = Rows(self.q, self.act, pad=self.pad_q), Rows(np.zeros((self.T, self.heads, self.latent)), self.act, pad=self.pad_o, filled=False)
        self.dtable, self.dlengths, self.dstarts = i32(self.table), i32(self.lengths), i32(self.starts)
        self.desc = G.make_latent_attention(
            q=self.dq.buf.data_ptr(), out=self.dout.buf.data_ptr(), table=self.dtable.data_ptr(), lengths=self.dlengths.data_ptr(),
            starts=self.dstarts.data_ptr(), ldq=self.dq.ld, ldo=self.dout.ld, table_width=self.table.shape[1], n_requests=len(self.fresh), T=self.T,
            heads=self.heads, max_fresh=max(1, max(self.fresh)) if max_fresh is None else max_fresh,
            max_length=max(1, max(self.lengths)) if max_length is None else max_length, scale=self.scale)
        self.ws = torch.full((G.glowq_latent_attention_workspace_bytes(self.dc.desc, self.desc),), 0xFF, dtype=torch.uint8, device="cuda")
        return self

    def run(self):
        G.glowq_latent_attention(self.dc.desc, self.desc, self.ws.data_ptr(), self.ws.numel(), stream())
        return self

    def output(self):
        rows = int(self.starts[-1])
        out = self.dout.numbers()
        assert np.isnan(out[rows:]).all(), "rows behind the last sequence were written"
        return out[:rows]

    def reference(self):
        rows = int(self.starts[-1])
        out, bound = np.zeros((rows, self.heads, self.latent)), np.zeros((rows, self.heads, self.latent))
        for r, n in enumerate(self.lengths):
            f = self.fresh[r]
            if f == 0:
                continue
            slots = L.slots_of(self.table, r, n, self.B, self.cache.n_blocks)
            lat = torch.from_numpy(self.cache.latents(slots)).cuda()
            k = torch.cat([lat, torch.from_numpy(self.cache.key_parts(slots)).cuda()], 1)
            e = torch.from_numpy(self.cache.exps[np.maximum(slots, 0)].astype(np.float64)).cuda()
            t = slice(int(self.starts[r]), int(self.starts[r]) + f)
            q = torch.from_numpy(self.q[t]).cuda().reshape(f * self.heads, -1)
            p = torch.arange(n - f, n, device="cuda").repeat_interleave(self.heads)[:, None]
            see = (torch.arange(max(n, 0), device="cuda")[None] <= p) & torch.from_numpy(slots >= 0).cuda()[None]
            o, b = softmax_reference(q, k, lat, see, self.scale, self.act, self.latent + self.rope, e)
            out[t], bound[t] = (x.cpu().numpy().reshape(f, self.heads, self.latent) for x in (o, b))
        return out, bound

    def check(self):
        return within(self.output(), *self.reference())


class Expanded:
    """Requests (cached, fresh) with rows of keys and values, a head's key beside its value."""

    def __init__(self, rng, requests, heads, nope, rope, act, q_scale=1.0, pad=0, gap=0, extra_rows=2, extra_keys=3, beside=True):
        self.act, self.heads, self.nope, self.rope = act, heads, nope, rope
        self.fresh, self.lengths = [f for _, f in requests], [c + f for c, f in requests]
        self.starts = np.concatenate([[0], np.cumsum(self.fresh)]).astype(int)
        n = np.maximum(self.lengths, 0)
        # requests' keys in another order than their rows
        order, at = rng.permutation(len(n)), 0
        self.key_starts = np.zeros(len(n), int)
        for r in order:
            self.key_starts[r] = at
            at += n[r]
        self.keys, self.T = max(1, at) + extra_keys, max(1, int(self.starts[-1])) + extra_rows
        self.q = act_round(rng.standard_normal((self.T, heads, nope + rope)) * q_scale, act)
        self.k, self.v = (act_round(rng.standard_normal((self.keys, heads, nope)), act) for _ in range(2))
        self.kr = act_round(rng.standard_normal((self.keys, rope)), act)
        for x in (self.k, self.v, self.kr):
            x[at:] = np.nan                                       # rows that no request has
        self.pad, self.gap, self.beside, self.scale = pad, gap, beside, 1.0 / math.sqrt(nope + rope)

    def device(self, max_fresh=None, max_length=None):
        N, act = self.nope, self.act
        self.dq, self.dout = Rows(self.q, act, self.gap, self.pad), Rows(np.zeros((self.T, self.heads, N)), act, 0, self.pad, filled=False)
        self.dr = Rows(self.kr[:, None], act, 0, self.pad)
        if self.beside:
            kv = Rows(np.concatenate([self.k, self.v], -1), act, self.gap, self.pad)
            self.dk = self.dv = kv
            v_at = kv.buf.data_ptr() + N * 2
        else:
            self.dk, self.dv = Rows(self.k, act, self.gap, self.pad), Rows(self.v, act, 0, 8)
            v_at = self.dv.buf.data_ptr()
        self.dstarts, self.dkey_starts, self.dlengths = i32(self.starts), i32(self.key_starts), i32(self.lengths)
        self.desc = G.make_expanded_attention(
            q=self.dq.buf.data_ptr(), k=self.dk.buf.data_ptr(), k_rope=self.dr.buf.data_ptr(), v=v_at, out=self.dout.buf.data_ptr(),
            starts=self.dstarts.data_ptr(), key_starts=self.dkey_starts.data_ptr(), lengths=self.dlengths.data_ptr(), ldq=self.dq.ld, lhq=self.dq.lh,
            ldk=self.dk.ld, lhk=self.dk.lh, ldr=self.dr.ld, ldv=self.dv.ld, lhv=self.dv.lh, ldo=self.dout.ld, n_requests=len(self.fresh), T=self.T,
            keys=self.keys, heads=self.heads, nope_dim=N, rope_dim=self.rope, v_dim=N, act_dtype=ACT_CODE[act],
            max_fresh=max(1, max(self.fresh)) if max_fresh is None else max_fresh,
            max_length=max(1, max(self.lengths)) if max_length is None else max_length, scale=self.scale)
        self.ws = torch.full((G.glowq_expanded_attention_workspace_bytes(self.desc),), 0xFF, dtype=torch.uint8, device="cuda")
        return self

    def run(self):
        G.glowq_expanded_attention(self.desc, self.ws.data_ptr(), self.ws.numel(), stream())
        return self

    def output(self):
        rows = int(self.starts[-1])
        out = self.dout.numbers()
        assert np.isnan(out[rows:]).all(), "rows behind the last sequence were written"
        return out[:rows]

    def reference(self):
        rows, N = int(self.starts[-1]), self.nope
        out, bound = np.zeros((rows, self.heads, N)), np.zeros((rows, self.heads, N))
        for r, n in enumerate(self.lengths):
            f, at = self.fresh[r], slice(int(self.key_starts[r]), int(self.key_starts[r]) + max(n, 0))
            if f == 0:
                continue
            t = slice(int(self.starts[r]), int(self.starts[r]) + f)
            see = torch.arange(max(n, 0), device="cuda")[None] <= torch.arange(n - f, n, device="cuda")[:, None]
            for h in range(self.heads):
                k = torch.from_numpy(np.concatenate([self.k[at, h], self.kr[at]], 1)).cuda()
                o, b = softmax_reference(torch.from_numpy(self.q[t, h]).cuda(), k, torch.from_numpy(self.v[at, h]).cuda().contiguous(), see, self.scale,
                                         self.act, N + self.rope)
                out[t, h], bound[t, h] = o.cpu().numpy(), b.cpu().numpy()
        return out, bound

    def check(self):
        return within(self.output(), *self.reference())


def within(got, want, bound):
    off = np.abs(got - want)
    bad = ~(off <= bound)
    assert not bad.any(), (int(bad.sum()), bad.size, float(np.nanmax(off / bound)), np.argwhere(bad)[:4].tolist())
    return got
