"""One decoder block's attention half while it serves: q/k/v group, cache, attention, o_proj.

    python examples/serve_block.py

A batch of requests of an 8B-sized block (32 heads of 128 over 8 key/value heads, random W4A16 weights without a
correction) comes in as prompts and then decodes token by token.  Every step is

    glowq_kv_plan            lengths -> tables, rows, slots   on the GPU
    glowq_group_forward      X -> q, k, v                     the framework's W4A16 maps
    glowq_kv_append_rotated  q and k with their positions;  k, v -> the 8-bit cache
    glowq_kv_attention       q over the cache -> X of o_proj
    glowq_group_forward      -> the block's output

all on one stream, with buffers that are made once.  At the end a request is served again with all its tokens as one prompt:
its rows agree with those of the steps up to the cache's grid.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_25385_amd as G

HIDDEN, HEADS, KV_HEADS, DIM, BLOCK = 4096, 32, 8, 128, 64
MAX_ROWS, MAX_REQUESTS, MAX_LENGTH, N_BLOCKS = 2048, 16, 4096, 256
DT, ACT = torch.bfloat16, G.GLOWQ_BF16


def stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class Linear:
    """An input-sharing group of W4A16 maps with random weights."""

    def __init__(self, d_in, d_outs, gen):
        self.d_in, self.d_outs, self.prepared = d_in, d_outs, []
        for o in d_outs:
            w = torch.randn(o, d_in, generator=gen, device="cuda") * 0.02
            wq = torch.empty(o, d_in // 8, dtype=torch.int32, device="cuda")
            sc, zp = (torch.empty(o, d_in // 128, dtype=torch.int16, device="cuda") for _ in range(2))
            G.glowq_quantize_rtn(w.data_ptr(), o, d_in, 128, wq.data_ptr(), sc.data_ptr(), zp.data_ptr(), stream())
            p = torch.empty(G.glowq_prepared_bytes(o, d_in, 128), dtype=torch.uint8, device="cuda")
            G.glowq_prepare_weights(wq.data_ptr(), sc.data_ptr(), zp.data_ptr(), o, d_in, 128, p.data_ptr(), stream())
            self.prepared.append(p)
        self.y = [torch.empty(MAX_ROWS, o, dtype=DT, device="cuda") for o in d_outs]
        self.ws = torch.empty(G.glowq_workspace_bytes([self.unit(self.y[0], MAX_ROWS)]), dtype=torch.uint8, device="cuda")
        G.glowq_workspace_init(self.ws.data_ptr(), self.ws.numel(), stream())

    def unit(self, x, T):
        mods = [G.make_module(p.data_ptr(), 0, y.data_ptr(), o, o) for p, y, o in zip(self.prepared, self.y, self.d_outs)]
        return G.make_unit(x.data_ptr(), 0, mods, T, self.d_in, 0, 128, ACT, ACT)

    def __call__(self, x, T):
        G.glowq_group_forward(self.unit(x, T), False, self.ws.data_ptr(), self.ws.numel(), stream())
        return [y[:T] for y in self.y]


class Server:
    """The weights, the cache, the requests' tables; the list of free blocks is the host's."""

    def __init__(self, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv, self.o = Linear(HIDDEN, [HEADS * DIM, KV_HEADS * DIM, KV_HEADS * DIM], gen), Linear(HEADS * DIM, [HIDDEN], gen)
        shape = G.make_kv_cache(0, 0, 0, 0, N_BLOCKS, BLOCK, KV_HEADS, DIM)
        codes, scales = G.glowq_kv_cache_bytes(shape)
        self.mem = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (codes, codes, scales, scales)]
        self.cache = G.make_kv_cache(*[m.data_ptr() for m in self.mem], N_BLOCKS, BLOCK, KV_HEADS, DIM)
        turns, magnitude = G.glowq_rope_turns(G.make_rope_spec(rotary_dim=DIM, scaling=G.GLOWQ_ROPE_PLAIN, base=10000.0, factor=1.0, low=0.0, high=0.0, trained_length=0))
        self.turns = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64, device="cuda")
        self.rope = G.make_rope(turns=self.turns.data_ptr(), rotary_dim=DIM, layout=G.GLOWQ_ROPE_HALVES, magnitude=magnitude)
        i32 = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")
        self.table, self.lengths, self.starts = i32(MAX_REQUESTS, MAX_LENGTH // BLOCK), i32(MAX_REQUESTS), i32(MAX_REQUESTS + 1)
        self.slots, self.positions, self.taken = i32(MAX_ROWS), i32(MAX_ROWS), i32(1)
        self.free = torch.randperm(N_BLOCKS, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.held = [0] * MAX_REQUESTS                     # tokens in the cache
        self.att = torch.empty(MAX_ROWS, HEADS * DIM, dtype=DT, device="cuda")
        self.ws = None

    def step(self, x, fresh):
        """x [rows][HIDDEN], fresh tokens of every request -> the block's rows after o_proj."""
        T, n = sum(fresh), len(fresh)
        cached = torch.tensor(self.held[:n], dtype=torch.int32).cuda()
        new = torch.tensor(fresh, dtype=torch.int32).cuda()
        plan = G.make_kv_step(cached=cached.data_ptr(), fresh=new.data_ptr(), free_blocks=self.free.data_ptr(), table=self.table.data_ptr(),
                              lengths=self.lengths.data_ptr(), starts=self.starts.data_ptr(), slots=self.slots.data_ptr(),
                              positions=self.positions.data_ptr(), taken=self.taken.data_ptr(), n_requests=n, n_free=self.free.numel(),
                              table_width=self.table.shape[1], max_tokens=T, block_tokens=BLOCK)
        G.glowq_kv_plan(plan, stream())
        q, k, v = self.qkv(x, T)
        rows = G.make_rope_rows(x=q.data_ptr(), y=q.data_ptr(), heads=HEADS, ldx=HEADS * DIM, lhx=DIM, ldy=HEADS * DIM, lhy=DIM)         # in place
        G.glowq_kv_append_rotated(self.cache, self.rope, rows, k.data_ptr(), KV_HEADS * DIM, v.data_ptr(), KV_HEADS * DIM, ACT,
                                  self.slots.data_ptr(), self.positions.data_ptr(), T, stream())
        att = G.make_kv_attention(q=q.data_ptr(), out=self.att.data_ptr(), table=self.table.data_ptr(), lengths=self.lengths.data_ptr(),
                                  starts=self.starts.data_ptr(), ldq=HEADS * DIM, ldo=HEADS * DIM, table_width=self.table.shape[1], n_requests=n,
                                  T=T, heads=HEADS, act_dtype=ACT, max_fresh=max(fresh),
                                  max_length=max(h + f for h, f in zip(self.held, fresh)), window=0, scale=1.0 / math.sqrt(DIM))
        need = G.glowq_kv_attention_workspace_bytes(self.cache, att)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            G.glowq_workspace_init(self.ws.data_ptr(), need, stream())
        G.glowq_kv_attention(self.cache, att, self.ws.data_ptr(), self.ws.numel(), stream())
        # the host knows the lengths, so it knows what the plan took
        taken = sum(-(-(h + f) // BLOCK) - -(-h // BLOCK) for h, f in zip(self.held, fresh))
        self.free = self.free[taken:].clone()
        for r, f in enumerate(fresh):
            self.held[r] += f
        return self.o(self.att, T)[0]


def main(prompts=(700, 33, 260), tokens=40) -> float:
    server = Server()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = [torch.randn(p + tokens, HIDDEN, generator=gen, device="cuda").to(DT) for p in prompts]      # every token's hidden row
    rows = [[] for _ in prompts]
    y = server.step(torch.cat([v[:p] for v, p in zip(x, prompts)]), list(prompts))
    for r, part in enumerate(y.split(list(prompts))):
        rows[r].append(part.clone())
    for t in range(tokens):
        y = server.step(torch.stack([v[p + t] for v, p in zip(x, prompts)]), [1] * len(prompts))
        for r in range(len(prompts)):
            rows[r].append(y[r:r + 1].clone())
    # the first request again, as one prompt
    again = Server()
    want = again.step(x[0], [x[0].shape[0]]).float()
    got = torch.cat(rows[0]).float()
    off = float((got - want).norm() / want.norm())
    print(f"{len(prompts)} prompts of {', '.join(map(str, prompts))} tokens, {tokens} steps: in steps and at once differ by {off:.1e}")
    return off


if __name__ == "__main__":
    main()
