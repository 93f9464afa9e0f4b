"""Glue for the tests of the serving operators: requests and an 8-bit cache drawn with numpy, moved to the GPU, and the
calls of the C ABI through the binding."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from gpu_util import ACT_CODE, TORCH_ACT, stream

ROUNDOFF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def act_round(x, act):
    """float64 numbers of the activation type nearest to x."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.float32).to(TORCH_ACT[act]).to(torch.float64).numpy()


class DeviceCache:
    """The bytes of an oracle cache on the GPU; what no request uses is filled with the NaN code."""

    def __init__(self, cache: K.Cache, used=None):
        self.o = cache
        self.codes, self.scales = [], []
        for w in range(2):
            codes, scales = cache.pages(w)
            if used is not None:
                at = K.places(cache.B, cache.D, w == 1)
                free = np.setdiff1d(np.arange(cache.n_blocks * cache.B), np.asarray(used))
                for s in free:
                    codes[s // cache.B][:, at[s % cache.B]] = 0xFF
            self.codes.append(torch.from_numpy(codes).cuda())
            self.scales.append(torch.from_numpy(scales).cuda())
        self.desc = G.make_kv_cache(self.codes[0].data_ptr(), self.codes[1].data_ptr(), self.scales[0].data_ptr(),
                                    self.scales[1].data_ptr(), cache.n_blocks, cache.B, cache.kv, cache.D)

    def tokens(self, w, slots):
        """Numbers of the device's tokens [len(slots)][kv][D], read from its bytes."""
        c = self.o
        codes, scales = self.codes[w].cpu().numpy(), self.scales[w].cpu().numpy().astype(np.int64)
        at = K.places(c.B, c.D, w == 1)
        out = np.empty((len(slots), c.kv, c.D))
        for i, s in enumerate(slots):
            b = int(s) // c.B
            out[i] = np.ldexp(K.VALUES[codes[b][:, at[int(s) % c.B]]], scales[b][:, None] - 127)
        return out


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def random_cache(rng, n_blocks, B, kv, D, spread=2):
    c = K.Cache(n_blocks, B, kv, D)
    for w in range(2):
        c.codes[w] = K.encode(np.clip(rng.standard_normal(c.codes[w].shape) * 72.0, -448, 448))
        c.exps[w] = rng.integers(-7 - spread, -6 + spread, c.exps[w].shape)
    return c


class Batch:
    """Requests (cached, fresh) over a random cache; the fresh tokens are in it already."""

    def __init__(self, rng, requests, heads, kv, D, B, act, spare=3, q_scale=1.0, pad_q=0, pad_o=0, extra_rows=2, spread=2):
        self.act, self.heads, self.kv, self.D, self.B = act, heads, kv, D, B
        self.fresh, self.lengths = [f for _, f in requests], [c + f for c, f in requests]
        self.starts = np.concatenate([[0], np.cumsum(self.fresh)])
        n = [max(0, -(-L // B)) for L in self.lengths]
        width = max(1, max(n))
        ids = rng.permutation(sum(n) + spare)
        self.table = np.full((len(requests), width), -1, np.int64)
        at = 0
        for r, k in enumerate(n):
            self.table[r, :k] = ids[at:at + k]
            at += k
        self.cache = random_cache(rng, sum(n) + spare, B, kv, D, spread)
        self.used = [int(self.table[r, j // B]) * B + j % B for r, L in enumerate(self.lengths) for j in range(max(L, 0))]
        self.T = max(1, int(self.starts[-1])) + extra_rows
        self.q = act_round(rng.standard_normal((self.T, heads, D)) * q_scale, act)
        self.pad_q, self.pad_o = pad_q, pad_o

    def device(self, max_fresh=None, max_length=None, window=0, scale=None):
        d = DeviceCache(self.cache, self.used)
        w = self.heads * self.D
        self.dq = torch.full((self.T, w + self.pad_q), float("nan"), dtype=TORCH_ACT[self.act], device="cuda")
        self.dq[:, :w] = torch.from_numpy(self.q.reshape(self.T, w)).to(TORCH_ACT[self.act]).cuda()
        self.dout = torch.full((self.T, w + self.pad_o), float("nan"), dtype=TORCH_ACT[self.act], device="cuda")
        self.dtable, self.dlengths, self.dstarts = i32(self.table), i32(self.lengths), i32(self.starts)
        self.scale = 1.0 / math.sqrt(self.D) if scale is None else scale
        self.window = window
        self.desc = G.make_kv_attention(
            q=self.dq.data_ptr(), out=self.dout.data_ptr(), table=self.dtable.data_ptr(), lengths=self.dlengths.data_ptr(),
            starts=self.dstarts.data_ptr(), ldq=w + self.pad_q, ldo=w + self.pad_o, table_width=self.table.shape[1],
            n_requests=len(self.fresh), T=self.T, heads=self.heads, act_dtype=ACT_CODE[self.act],
            max_fresh=max(1, max(self.fresh)) if max_fresh is None else max_fresh,
            max_length=max(1, max(self.lengths)) if max_length is None else max_length, window=window, scale=self.scale)
        self.ws = torch.empty(G.glowq_kv_attention_workspace_bytes(d.desc, self.desc), dtype=torch.uint8, device="cuda")
        G.glowq_workspace_init(self.ws.data_ptr(), self.ws.numel(), stream())
        self.dc = d
        return self

    def run(self):
        G.glowq_kv_attention(self.dc.desc, self.desc, self.ws.data_ptr(), self.ws.numel(), stream())
        return self

    def output(self):
        """[starts[-1]][heads][D]; what no row covers must be untouched."""
        torch.cuda.synchronize()
        rows, w = int(self.starts[-1]), self.heads * self.D
        assert torch.isnan(self.dout[rows:]).all() and torch.isnan(self.dout[:, w:]).all()
        return self.dout[:rows, :w].double().cpu().numpy().reshape(rows, self.heads, self.D)

    def reference(self, q=None):
        """(out, bound) in 64 bits.  The bound on |error|: weights rounded to the activation type and the result's own
        rounding, u each of sum p |V| and |out|; scores in fp32, their sums off by (D + 4) 2^-24 sum |q k| scale at most,
        in the weights and in their sum; sums over L keys; the exponential's last places; weights below the normal range of
        binary16, off by 2^-25 of the largest block's grid."""
        q = self.q if q is None else q
        u, group, D = ROUNDOFF[self.act], self.heads // self.kv, self.D
        rows = int(self.starts[-1])
        out, bound = np.zeros((rows, self.heads, D)), np.zeros((rows, self.heads, D))
        for r, L in enumerate(self.lengths):
            f = self.fresh[r]
            if f == 0:
                continue
            e = self.table[r][np.arange(max(L, 0)) // self.B]
            there = (e >= 0) & (e < self.cache.n_blocks)
            slots = np.where(there, e * self.B + np.arange(max(L, 0)) % self.B, -1)
            Kt, Vt = (torch.from_numpy(self.cache.tokens(w, slots)).cuda() for w in range(2))
            qr = torch.from_numpy(q[int(self.starts[r]):int(self.starts[r]) + f]).cuda()
            p = torch.arange(L - f, L, device="cuda")[:, None]
            j = torch.arange(max(L, 0), device="cuda")[None]
            see = (j <= p) & torch.from_numpy(there).cuda()[None]
            if self.window:
                see &= j > p - self.window
            none = ~see.any(1)
            for h in range(self.heads):
                k, v = Kt[:, h // group], Vt[:, h // group]
                s = (qr[:, h] @ k.T.contiguous() * self.scale).masked_fill(~see, -math.inf)
                w = torch.softmax(s, 1)
                w[none] = 0.0
                size = (qr[:, h].abs() @ k.abs().T.contiguous() * self.scale).masked_fill(~see, 0.0).amax(1, keepdim=True) if L > 0 else 0.0
                o, mag = w @ v.contiguous(), w @ v.abs().contiguous()
                # (hidden numbers that are none must not show: they are held to by the caller)
                top = (v.abs().amax(1)[None] * see).amax(1, keepdim=True) if L > 0 else 0.0
                eps = 2.0 ** -24 * (2 * (D + 4) * size + 2 * L + 64)
                t = slice(int(self.starts[r]), int(self.starts[r]) + f)
                out[t, h] = o.cpu().numpy()
                small = L * 2.0 ** -25 * top if self.act == "f16" else 0.0
                bound[t, h] = ((u + eps) * mag + u * o.abs() + small + 2.0 ** -24).cpu().numpy()
        return out, bound

    def check(self, q=None):
        got = self.output()
        out, bound = self.reference(q)
        off = np.abs(got - out)
        bad = ~(off <= bound)
        assert not bad.any(), (int(bad.sum()), bad.size, float(np.nanmax(off / bound)), np.argwhere(bad)[:4].tolist())
        return got
