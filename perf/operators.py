"""The serving operators between a block's q/k/v group and its o_proj, timed: block tables and
slot maps from request lengths, new tokens into an 8-bit cache of keys and values, attention
that reads this cache; alone and as one step of a serving program.

The cache.  Requests hold their tokens in blocks of `block` tokens, found through a table
[request][width].  A block of one head is a page of `block * D` E4M3 codes with one scale
2^(byte - 127), for keys and for values:
    scale exponent  e = the smallest with max |x| <= 448 * 2^e over the block's tokens of the
                    head (finite ones; at least -64),
    code            x * 2^-e rounded to E4M3, ties to even;
a block that gets more tokens later keeps its exponent or takes a larger one, and then its
older tokens are rounded to the new grid.  Pages are stored in 16-token tiles, 64 dims a piece:
keys  [block / 16][D / 64][4 groups of 16 dims][16 tokens][16 dims],
values [block / 16][D / 64][4 groups of 4 tokens][16 dims][4 pieces of 16 dims][4 tokens].

Attention of new token i of a request with `fresh` new ones and `length` in all, for q head h
(its key/value head is h // (heads / kv_heads)):
    p = length - fresh + i,  keys j with max(0, p - window + 1) <= j <= p,
    out = sum_j softmax_j(q . K_j / sqrt(D)) V_j,   K and V as the cache holds them.

Head layouts and widths are those of the repository's decoder blocks (32 heads of 128 with 8
or 32 key/value heads, 40 heads), and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

ACT = {"f16": torch.float16, "bf16": torch.bfloat16}
EMIN = -64
GOLDEN = 0.6180339887498949


# ---- cases ------------------------------------------------------------------------------
def plan(ones, prompts, new, old, block, pad=1):
    """Tables and slots of a step: `ones` requests with one new token, `prompts` with up to
    `new`, up to `old` tokens cached already; slot maps padded to a multiple of `pad`."""
    return {"kind": "plan", "ones": ones, "prompts": prompts, "new": new, "old": old, "block": block, "pad": pad}


def cache_case(kind, ones, prompts, new, old, heads, kv_heads, D, block, act, window=0):
    return {"kind": kind, "ones": ones, "prompts": prompts, "new": new, "old": old, "block": block, "pad": 1,
            "heads": heads, "kv_heads": kv_heads, "D": D, "act": act, "window": window}


def listed():
    return [
        # tables of 64 sequences that decode, one token each
        dict(plan(64, 0, 1, 8000, 64), name="plan_n64"),
        # a prompt phase of many users: 300 prompts beside 700 decoding sequences, padded slot map
        dict(plan(700, 300, 1000, 4000, 16, pad=256), name="plan_n1000"),
        # 64 decoding sequences put one token each into the cache, 8 key/value heads
        dict(cache_case("append", 64, 0, 1, 8000, 32, 8, 128, 64, "f16"), name="append_n64"),
        # four ragged prompts into the cache, 32 key/value heads, the last blocks partly filled before
        dict(cache_case("append", 0, 4, 2100, 100, 32, 32, 128, 32, "bf16"), name="append_prompts_bf16"),
        # one sequence, early in its answer: what a call costs
        dict(cache_case("attend", 1, 0, 1, 900, 32, 8, 128, 64, "f16"), name="attend_n1"),
        # 64 sequences decoding at ragged lengths up to 8000, grouped heads
        dict(cache_case("attend", 64, 0, 1, 8000, 32, 8, 128, 64, "bf16"), name="attend_n64_bf16"),
        # 17 sequences of a 13B-sized model, every head with its own keys, small blocks
        dict(cache_case("attend", 17, 0, 1, 3900, 40, 40, 128, 16, "f16"), name="attend_n17_mha"),
        # two very long documents, one token at a time
        dict(cache_case("attend", 2, 0, 1, 131000, 32, 8, 128, 128, "f16"), name="attend_long"),
        # pieces of three prompts on what is cached of them, sliding window
        dict(cache_case("attend", 0, 3, 500, 16000, 32, 8, 128, 64, "f16", window=4096), name="attend_pieces"),
        # one long prompt
        dict(cache_case("attend", 0, 1, 8000, 0, 32, 8, 128, 64, "bf16"), name="attend_prompt_bf16"),
        # heads of 64: a prompt of 1500 tokens comes in beside 40 decoding sequences
        dict(cache_case("attend", 40, 1, 1500, 2000, 16, 4, 64, 32, "bf16"), name="attend_mixed_d64"),
        # a whole decoding step of 32 sequences: tables, cache, attention
        dict(cache_case("step", 32, 0, 1, 2000, 32, 8, 128, 64, "bf16"), name="step_n32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "attend", "step"])
    block = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        prompts = rng.choice([0, 0, _log(rng, 1, 300)])
        return plan(_log(rng, 1, 700), prompts, _log(rng, 2, 1000), _log(rng, 1, 8000), block, rng.choice([1, 64, 256]))
    heads, kv = rng.choice([(32, 8), (32, 32), (40, 40), (28, 4), (16, 2), (24, 8), (20, 20)])
    D, act = rng.choice([64, 128, 128]), rng.choice(["f16", "bf16"])
    window = rng.choice([0, 0, 0, _log(rng, 100, 5000)]) if kind == "attend" else 0
    if kind == "append":
        if rng.random() < 0.5:
            return cache_case(kind, _log(rng, 1, 128), 0, 1, _log(rng, 1, 8000), heads, kv, D, block, act)
        return cache_case(kind, 0, rng.randint(1, 4), _log(rng, 2, 2100), _log(rng, 1, 2000), heads, kv, D, block, act)
    how = "ones" if kind == "step" else rng.choice(["ones", "ones", "pieces", "prompts", "mixed"])
    if how in ("ones", "mixed"):
        ones = _log(rng, 1, 64)
        old = _log(rng, 1, max(2, min(131000, int(0.9e9 / (ones * kv * D * 2)))))
        if kind == "step":
            old = min(old, 8000)
        if how == "ones":
            return cache_case(kind, ones, 0, 1, old, heads, kv, D, block, act, window)
        return cache_case(kind, ones, 1, _log(rng, 2, 2500), min(old, 8000), heads, kv, D, block, act, window)
    prompts = rng.randint(1, 4)
    old = _log(rng, 100, 30000) if how == "pieces" else 0
    new = _log(rng, 2, 1000) if how == "pieces" else _log(rng, 2, 5500)
    while prompts * heads * new * (old + new) > 1.0e9:
        new, old = max(2, new // 2), old // 2
    return cache_case(kind, 0, prompts, new, old, heads, kv, D, block, act, window)


def _requests(case):
    """(fresh, cached) of every request: prompts first, lengths spread evenly over their range."""
    fresh, cached = [], []
    for i in range(case["prompts"]):
        f = (i * GOLDEN) % 1.0
        fresh.append(max(1, int(case["new"] * (1.0 - 0.7 * f))))
        cached.append(int(case["old"] * (1.0 - 0.8 * ((i * GOLDEN + 0.3) % 1.0))) if case["old"] else 0)
    for i in range(case["ones"]):
        fresh.append(1)
        cached.append(int(case["old"] * (1.0 - 0.9 * ((i * GOLDEN) % 1.0))))
    return fresh, cached


def work(case):
    fresh, cached = _requests(case)
    T, n, B = sum(fresh), len(fresh), case["block"]
    by = fl = 0.0
    if case["kind"] in ("plan", "step"):
        new = sum(-(-(c + f) // B) - -(-c // B) for f, c in zip(fresh, cached))
        # lengths in; table entries of the tokens' blocks in or out, new blocks' ids in; per token slot and position out
        by += n * 8 + T * 8 + n * 8 + sum(-(-(c + f) // B) - c // B for f, c in zip(fresh, cached)) * 4 + new * 4
    if case["kind"] == "plan":
        return {"bytes": by, "flops": 0}
    kv, D = case["kv_heads"], case["D"]
    if case["kind"] in ("append", "step"):
        # keys and values in, codes out, scales
        blocks = sum(-(-(c + f) // B) - c // B for f, c in zip(fresh, cached))
        by += T * kv * D * 2 * 2 + T * kv * D * 2 + T * 4 + blocks * kv * 2
        if case["kind"] == "append":
            # ... and read back: the tokens of the blocks that were touched
            rows = sum((c + f) - c // B * B for f, c in zip(fresh, cached))
            by += rows * kv * D * 2 * (1 + 2)
            return {"bytes": by, "flops": 0}
    h, w = case["heads"], case["window"]
    by += T * h * D * 2 * 2
    for f, c in zip(fresh, cached):
        lo = max(0, c - w + 1) if w else 0
        by += (c + f - lo) * kv * (D * 2 + 2.0 / B)
        first, last = c + 1, c + f                           # visible keys of the first and the last new token
        if not w or last <= w:
            pairs = (first + last) * f / 2
        elif first >= w:
            pairs = f * w
        else:
            pairs = (first + w) * (w - first + 1) / 2 + (last - w) * w
        fl += 4.0 * D * h * pairs
    return {"bytes": by, "flops": fl}


# ---- inputs -----------------------------------------------------------------------------
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    perm = torch.Generator().manual_seed(seed)
    fresh, cached = _requests(case)
    p, n, B = case["prompts"], len(fresh), case["block"]
    order = torch.randperm(p, generator=perm).tolist() + [p + i for i in torch.randperm(n - p, generator=perm).tolist()]
    fresh, cached = [fresh[i] for i in order], [cached[i] for i in order]
    T = sum(fresh)
    had = [-(-c // B) for c in cached]
    has = [-(-(c + f) // B) for f, c in zip(fresh, cached)]
    width, total = max(has), sum(has)
    n_blocks = total + total // 8 + 1                         # a pool with a little more than is used
    ids = torch.randperm(n_blocks, generator=perm).to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32)
    first = 0
    for r in range(n):
        table[r, :had[r]] = ids[first:first + had[r]]
        first += had[r]
    s = {"case": case, "n": n, "T": T, "width": width, "n_blocks": n_blocks,
         "fresh": _i32(fresh), "cached": _i32(cached), "table": table.cuda(), "free": ids[first:].cuda()}
    s["max_new"], s["max_length"] = max(fresh), max(f + c for f, c in zip(fresh, cached))
    s["slots_T"] = -(-T // case["pad"]) * case["pad"]
    for name, size in (("lengths", n), ("starts", n + 1), ("slots", s["slots_T"]), ("positions", s["slots_T"]), ("taken", 1)):
        s[name] = torch.empty(size, dtype=torch.int32, device="cuda")
    if case["kind"] != "plan":
        _prepare_cache(s, case, gen, fresh, cached, had, has, ids)
    if own:
        _prepare_own(s)                                       # descriptors and the workspace that a program keeps
    return s


def _prepare_cache(s, case, gen, fresh, cached, had, has, ids):
    B, kv, D, h, T, n = case["block"], case["kv_heads"], case["D"], case["heads"], s["T"], s["n"]
    dt = ACT[case["act"]]

    def codes():
        # cached tokens: normal, codes up to 448
        c = torch.empty(s["n_blocks"], kv, B * D, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (kv * B * D))
        for b in range(0, s["n_blocks"], step):
            x = torch.randn(c[b:b + step].shape, generator=gen, device="cuda") * 72.0
            c[b:b + step] = x.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        return c

    # heads differ in magnitude, blocks of a head by a factor of two now and then
    def exponents(centre):
        head = torch.randint(centre - 1, centre + 2, (1, kv), generator=gen, device="cuda")
        return (127 + head + (torch.rand(s["n_blocks"], kv, generator=gen, device="cuda") < 0.2)).to(torch.uint8)

    s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"] = codes(), codes(), exponents(-6), exponents(-7)

    def fresh_rows(heads, scales):
        x = torch.randn(T, heads, D, generator=gen, device="cuda")
        return (x * (scales[:1].float() - 127.0).exp2().view(1, -1, 1) * 72.0).to(dt)

    s["k"], s["v"] = fresh_rows(kv, s["k_scales"]), fresh_rows(kv, s["v_scales"])
    s["q"] = (torch.randn(T, h, D, generator=gen, device="cuda") * 1.5).to(dt)
    s["out"] = torch.empty(T, h, D, dtype=dt, device="cuda")
    if case["kind"] == "step":
        return
    # the step's tables are at hand: new blocks taken from the pool in order
    first = sum(had)
    slots, touched = [], []
    for r in range(n):
        s["table"][r, had[r]:has[r]] = ids[first:first + has[r] - had[r]].cuda()
        first += has[r] - had[r]
    rows = s["table"].cpu()
    for r in range(n):
        at = torch.arange(cached[r] // B * B, cached[r] + fresh[r])
        at = rows[r][at // B].long() * B + at % B
        touched.append(at)
        slots.append(at[cached[r] % B:])
    s["slots"] = torch.cat(slots).to(torch.int32).cuda()
    s["touched"] = torch.cat(touched).to(torch.int32).cuda()
    s["lengths"] = s["cached"] + s["fresh"]
    s["starts"] = torch.nn.functional.pad(s["fresh"].cumsum(0), (1, 0)).to(torch.int32)
    if case["kind"] == "append":
        s["k_back"] = torch.empty(s["touched"].numel(), kv, D, dtype=dt, device="cuda")
        s["v_back"] = torch.empty_like(s["k_back"])


# ---- the framework's operators ----------------------------------------------------------
def _prepare_own(s):
    import paper_2603_25385_amd as G

    c = s["case"]
    s["G"] = G
    if c["kind"] in ("plan", "step"):
        s["step"] = G.make_kv_step(
            cached=s["cached"].data_ptr(), fresh=s["fresh"].data_ptr(), free_blocks=s["free"].data_ptr(),
            table=s["table"].data_ptr(), lengths=s["lengths"].data_ptr(), starts=s["starts"].data_ptr(),
            slots=s["slots"].data_ptr(), positions=s["positions"].data_ptr(), taken=s["taken"].data_ptr(),
            n_requests=s["n"], n_free=s["free"].numel(), table_width=s["width"], max_tokens=s["slots_T"],
            block_tokens=c["block"])
    if c["kind"] == "plan":
        return
    s["act"] = G.GLOWQ_F16 if c["act"] == "f16" else G.GLOWQ_BF16
    s["cache"] = G.make_kv_cache(s["k_codes"].data_ptr(), s["v_codes"].data_ptr(), s["k_scales"].data_ptr(),
                                 s["v_scales"].data_ptr(), s["n_blocks"], c["block"], c["kv_heads"], c["D"])
    if c["kind"] in ("attend", "step"):
        s["att"] = G.make_kv_attention(
            q=s["q"].data_ptr(), out=s["out"].data_ptr(), table=s["table"].data_ptr(), lengths=s["lengths"].data_ptr(),
            starts=s["starts"].data_ptr(), ldq=c["heads"] * c["D"], ldo=c["heads"] * c["D"], table_width=s["width"],
            n_requests=s["n"], T=s["T"], heads=c["heads"], act_dtype=s["act"], max_fresh=s["max_new"],
            max_length=s["max_length"], window=c["window"], scale=1.0 / math.sqrt(c["D"]))
        s["ws"] = torch.empty(G.glowq_kv_attention_workspace_bytes(s["cache"], s["att"]), dtype=torch.uint8, device="cuda")
        G.glowq_workspace_init(s["ws"].data_ptr(), s["ws"].numel(), torch.cuda.current_stream().cuda_stream)


def _run_own(s):
    c, G = s["case"], s["G"]
    st = torch.cuda.current_stream().cuda_stream
    out = {}
    if c["kind"] in ("plan", "step"):
        G.glowq_kv_plan(s["step"], st)
        out = {k: s[k] for k in ("table", "lengths", "starts", "slots", "positions", "taken")}
    if c["kind"] in ("append", "step"):
        ld = c["kv_heads"] * c["D"]
        G.glowq_kv_append(s["cache"], s["k"].data_ptr(), ld, s["v"].data_ptr(), ld, s["act"], s["slots"].data_ptr(), s["T"], st)
        if c["kind"] == "append":
            G.glowq_kv_gather(s["cache"], s["touched"].data_ptr(), s["touched"].numel(), s["k_back"].data_ptr(), ld,
                              s["v_back"].data_ptr(), ld, s["act"], st)
            out = {"k": s["k_back"], "v": s["v_back"]}
    if c["kind"] in ("attend", "step"):
        G.glowq_kv_attention(s["cache"], s["att"], s["ws"].data_ptr(), s["ws"].numel(), st)
        out["out"] = s["out"]
    return out


# ---- their plain forms ------------------------------------------------------------------
def _plain_plan(s):
    B, T = s["case"]["block"], s["slots_T"]
    cached, fresh = s["cached"].long(), s["fresh"].long()
    lengths = cached + fresh
    starts = torch.nn.functional.pad(fresh.cumsum(0), (1, 0))
    had, has = (cached + B - 1) // B, (lengths + B - 1) // B
    taken = (has - had).cumsum(0)
    t = torch.arange(T, device="cuda")
    live = t < starts[-1]
    r = (torch.searchsorted(starts, t, right=True) - 1).clamp(max=s["n"] - 1)
    pos = cached[r] + t - starts[r]
    b = (pos // B).clamp(max=s["width"] - 1)
    new = (taken - (has - had))[r] + b - had[r]
    block = torch.where(b >= had[r], s["free"][new.clamp(0, s["free"].numel() - 1)], s["table"][r, b])
    table = s["table"].clone()
    table[r[:s["T"]], b[:s["T"]]] = block[:s["T"]]
    none = torch.full_like(t, -1)
    return {"table": table, "lengths": lengths.int(), "starts": starts.int(), "taken": taken[-1:].int(),
            "slots": torch.where(live, block.long() * B + pos % B, none).int(), "positions": torch.where(live, pos, none).int()}


def _pow2(e):
    """2^e in 32 bits, by the exponent's place (a power function may be off in its last bit)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _round(x, e):
    """x on the grid of E4M3 codes times 2^e."""
    return (x * _pow2(-e)).to(torch.float8_e4m3fn).float() * _pow2(e)


def _exponent(top):
    m, x = torch.frexp(top / 448.0)                           # top / 448 = m 2^x, m in [1/2, 1)
    x = torch.where(m == 0.5, x - 1, x)
    return torch.where(top > 0, x, torch.full_like(x, EMIN)).clamp(min=EMIN)


def _tokens(pages, values, B, D):
    """Pages [..., B * D] as tokens [..., B, D] in 32 bits."""
    x, lead = pages.view(torch.float8_e4m3fn).float(), pages.shape[:-1]
    k = len(lead)
    if values:
        x = x.view(*lead, B // 16, D // 64, 4, 16, 4, 4).permute(*range(k), k, k + 2, k + 5, k + 1, k + 4, k + 3)
    else:
        x = x.view(*lead, B // 16, D // 64, 4, 16, 16).permute(*range(k), k, k + 3, k + 1, k + 2, k + 4)
    return x.reshape(*lead, B, D)


def _block_exponents(s, x, scales, slots):
    """The exponents [n_blocks][kv_heads] once x [T][kv_heads][D] is in the cache."""
    B, kv = s["case"]["block"], s["case"]["kv_heads"]
    block, at = slots.long() // B, slots.long() % B
    top = torch.where(x.isfinite(), x, torch.zeros_like(x)).abs().amax(-1)
    most = torch.zeros(s["n_blocks"], kv, device="cuda").index_reduce_(0, block, top, "amax")
    first = torch.full((s["n_blocks"],), B, device="cuda").index_reduce_(0, block, at, "amin")[:, None]
    e, before = _exponent(most), scales.int() - 127
    return torch.where(first == B, before, torch.where(first > 0, torch.maximum(before, e), e))


def _plain_append(s, name):
    """The tokens `touched`, as the cache holds them afterwards."""
    B, D, slots, back = s["case"]["block"], s["case"]["D"], s["slots"].long(), s["touched"].long()
    x = s[name].float()
    after = _block_exponents(s, x, s[name + "_scales"], slots)
    new = _round(x, after[slots // B].unsqueeze(-1))
    of = torch.full((s["n_blocks"] * B,), -1, device="cuda")
    of[slots] = torch.arange(s["T"], device="cuda")
    of = of[back]
    old = _tokens(s[name + "_codes"][back // B], name == "v", B, D).gather(
        2, (back % B).view(-1, 1, 1, 1).expand(-1, s["case"]["kv_heads"], 1, D)).squeeze(2)
    old = old * _pow2(s[name + "_scales"].int()[back // B].unsqueeze(-1) - 127)
    old = _round(old, after[back // B].unsqueeze(-1))
    return torch.where((of >= 0).view(-1, 1, 1), new[of.clamp(min=0)], old).to(ACT[s["case"]["act"]])


def _dense(s, name, table, scales, D):
    """Keys or values of all requests [n][kv_heads][width * block][D]."""
    B = s["case"]["block"]
    at = table.long().clamp(min=0)
    x = _tokens(s[name + "_codes"][at], name == "v", B, D)                             # [n][width][kv][B][D]
    x = x * _pow2(scales[at] - 127).view(*at.shape, -1, 1, 1)
    return x.permute(0, 2, 1, 3, 4).reshape(at.shape[0], -1, at.shape[1] * B, D)


def _plain_attend(c, lengths, fresh, q, k, v):
    """Rows q [n][new][heads][D], the first `fresh` of each request its new tokens; keys and values of all its tokens."""
    n, new, h, D = q.shape
    kv, L = c["kv_heads"], k.shape[2]
    q = q.float().view(n, new, kv, h // kv, D).permute(0, 2, 3, 1, 4).reshape(n, kv, h // kv * new, D).contiguous()
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(n, kv, h // kv, new, L)
    p = (lengths - fresh).view(n, 1) + torch.arange(new, device="cuda")
    j = torch.arange(L, device="cuda")
    seen = j <= p[..., None]
    if c["window"]:
        seen = seen & (j > p[..., None] - c["window"])
    x = x.masked_fill_(~seen.view(n, 1, 1, new, L), -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    x = x.div_(x.sum(-1, keepdim=True))
    x = torch.matmul(x.view(n, kv, h // kv * new, L), v)
    return x.view(n, kv, h // kv, new, D).permute(0, 3, 1, 2, 4).reshape(n, new, h, D)


def _plain_attend_all(s, lengths, keys):
    """Prompts, as a padded batch, and requests with one new token, as another."""
    c, p = s["case"], s["case"]["prompts"]
    q, fresh, starts = s["q"], s["fresh"].long(), torch.nn.functional.pad(s["fresh"].long().cumsum(0), (1, 0))
    out = torch.empty(s["T"] + 1, *q.shape[1:], device="cuda")                         # the row behind takes the padding
    if p:
        k, v = keys(slice(0, p))
        row = starts[:p, None] + torch.arange(s["max_new"], device="cuda")
        live = row < starts[1:p + 1, None]
        o = _plain_attend(c, lengths[:p], fresh[:p], q[row.clamp(max=s["T"] - 1)], k, v)
        out[torch.where(live, row, s["T"])] = o
    if c["ones"]:
        k, v = keys(slice(p, s["n"]))
        out[s["T"] - c["ones"]:s["T"]] = _plain_attend(c, lengths[p:], fresh[p:], q[s["T"] - c["ones"]:, None], k, v)[:, 0]
    return out[:s["T"]].to(ACT[c["act"]])


def _plain_step(s):
    """Tables, then the cache with the new tokens in it, then attention."""
    c = s["case"]
    B, D, T = c["block"], c["D"], s["T"]
    out = _plain_plan(s)
    slots, table, lengths = out["slots"].long(), out["table"], out["lengths"].long()
    r = torch.searchsorted(out["starts"], torch.arange(T, device="cuda"), right=True) - 1
    at = out["positions"].long()

    def one(name):
        x = s[name].float()
        after = _block_exponents(s, x, s[name + "_scales"], slots)
        dense = _dense(s, name, table, s[name + "_scales"].int(), D)
        e = after[table.long().clamp(min=0)]                                            # [n][width][kv]
        e = e.permute(0, 2, 1).repeat_interleave(B, dim=2).unsqueeze(-1)
        dense = _round(dense, e)
        dense[r, :, at] = _round(x, after[slots // B].unsqueeze(-1))
        # what lies behind a request's tokens may not even be a number
        behind = torch.arange(dense.shape[2], device="cuda") >= lengths[:, None]
        return dense.masked_fill_(behind[:, None, :, None], 0.0)

    k, v = one("k"), one("v")
    out["out"] = _plain_attend_all(s, lengths, lambda which: (k[which].contiguous(), v[which].contiguous()))
    return out


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s)
    if kind == "plan":
        return _plain_plan(s)
    if kind == "append":
        return {"k": _plain_append(s, "k"), "v": _plain_append(s, "v")}
    if kind == "step":
        return _plain_step(s)
    D = s["case"]["D"]
    return {"out": _plain_attend_all(
        s, s["lengths"].long(),
        lambda which: tuple(_dense(s, x, s["table"][which], s[x + "_scales"].int(), D) for x in ("k", "v")))}


# ---- the definition in 64 bits ----------------------------------------------------------
def _grid():
    """The value of every E4M3 code."""
    v = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = math.nan if c & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v.append(-x if c & 128 else x)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _places(B, D, values):
    """Byte of token t, dim d in a page, [B][D]."""
    t, d = torch.arange(B, device="cuda").view(-1, 1), torch.arange(D, device="cuda").view(1, -1)
    piece = (t // 16 * (D // 64) + d // 64) * 1024
    if values:
        return piece + (t % 16 // 4 * 16 + d % 16) * 16 + d % 64 // 16 * 4 + t % 4
    return piece + (d % 64 // 16 * 16 + t % 16) * 16 + d % 16


def _two_to(e):
    """2^e in 64 bits, exactly, for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x, e):
    """x rounded to the codes' grid times 2^e: steps of 2^(floor(log2 |x|) - 3), 2^(e - 9) at least."""
    floor = (x.abs().clamp(min=2.0 ** -300).view(torch.int64) >> 52) - 1023
    step = _two_to(torch.maximum(floor, e.long() - 6) - 3)
    return torch.round(x / step) * step


class _Held:
    """Keys or values of a request, token by token, from the pages, and with new tokens in them."""

    def __init__(self, s, name):
        self.s, self.name, self.grid = s, name, _grid()
        self.where = _places(s["case"]["block"], s["case"]["D"], name == "v")

    def tokens(self, row, fresh=0, length=0, start=0, new=False):
        """[length][kv_heads][D]; with `new`, the last `fresh` come from the step's rows."""
        s, B = self.s, self.s["case"]["block"]
        blocks = row[:-(-length // B)].long()
        held = self.grid[s[self.name + "_codes"][blocks].long()][..., self.where]       # [blocks][kv][B][D]
        e = s[self.name + "_scales"][blocks].long() - 127
        x = held * _two_to(e)[..., None, None]
        if new:
            c = length - fresh
            rows = s[self.name][start:start + fresh].double()
            for b in range(c // B, len(blocks)):
                lo, hi = max(c, b * B), min(length, (b + 1) * B)
                top = rows[lo - c:hi - c].abs().amax((0, 2))                            # [kv]
                grown = (top / 448.0 - 1e-12 * top).clamp(min=2.0 ** -300).view(torch.int64) >> 52
                need = (grown - 1022).clamp(min=EMIN)                                   # ceil(log2(top / 448))
                now = torch.maximum(need, e[b]) if lo > b * B else need
                x[b] = _nearest(x[b], now[:, None, None])
                x[b][:, lo - b * B:hi - b * B] = _nearest(rows[lo - c:hi - c], now[None, :, None]).permute(1, 0, 2)
        return x.permute(0, 2, 1, 3).reshape(len(blocks) * B, *x.shape[1::2])[:length]


def exact(case, seed):
    s = prepare(case, seed)
    kind, B, w = case["kind"], case["block"], case.get("window", 0)
    if kind == "plan":
        return None                                           # whole numbers throughout
    fresh, cached = s["fresh"].tolist(), s["cached"].tolist()
    table, free, first = s["table"].clone(), s["free"], 0
    if kind == "step":
        for r in range(s["n"]):
            had, has = -(-cached[r] // B), -(-(cached[r] + fresh[r]) // B)
            table[r, had:has] = free[first:first + has - had]
            first += has - had
    held, start, outs = {x: _Held(s, x) for x in ("k", "v")}, 0, {"k": [], "v": [], "out": []}
    for r in range(s["n"]):
        f, L = fresh[r], fresh[r] + cached[r]
        k, v = (held[x].tokens(table[r], f, L, start, kind != "attend") for x in ("k", "v"))
        if kind == "append":
            outs["k"].append(k[cached[r] // B * B:])
            outs["v"].append(v[cached[r] // B * B:])
        else:
            q, group = s["q"][start:start + f].double(), case["heads"] // case["kv_heads"]
            o = torch.empty_like(q)
            p = torch.arange(L - f, L, device="cuda")[:, None]
            j = torch.arange(L, device="cuda")
            hidden = (j > p) | (j <= p - w) if w else j > p
            for h in range(case["heads"]):
                x = q[:, h] @ k[:, h // group].t().contiguous() / math.sqrt(case["D"])
                o[:, h] = torch.softmax(x.masked_fill_(hidden, -math.inf), -1) @ v[:, h // group].contiguous()
            outs["out"].append(o)
        start += f
    if kind == "append":
        return {x: torch.cat(outs[x]) for x in ("k", "v")}
    out = {"out": torch.cat(outs["out"])}
    if kind == "step":
        out.update({k: None for k in ("table", "lengths", "starts", "slots", "positions", "taken")})
    return out
