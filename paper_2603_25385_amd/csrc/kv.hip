// The 8-bit cache of keys and values: block tables and slot maps of a step, new tokens into the cache, tokens read back.
#include <algorithm>
#include "kv_append.hpp"
#include "kv_host.hpp"

namespace glowq {

// ---------------------------------------------------------------------------------------
// Tables and slots of a step.  Two running sums over the requests (tokens, blocks) and one look-up per token; the work is
// a few bytes per token, so the launch and its chain of dependent loads are the time (64 requests 4.7 us, 1000 with 196000
// tokens 8.2).  Every workgroup adds up all requests itself (8 bytes each, from the L2 after the first) rather than waiting for
// one that does: one launch, nothing to hand over.  The sums before every request, or every few where they are many, lie in
// LDS; a thread finds its first token's request by bisection there and goes on from it for the next three.
constexpr int PLAN_THREADS = 256;
constexpr int PLAN_TOKENS = 4;         // per thread, one after another
constexpr int PLAN_SHARES = 4096;

struct PlanArgs {
  const int32_t *cached, *fresh, *free_blocks;
  int32_t *table, *lengths, *starts, *slots, *positions, *taken;
  int n, n_free, width, max_tokens, block_shift;
  int share, shares;                   // requests of a share, shares in all
};

__device__ inline long long plan_blocks(long long tokens, const PlanArgs& a) {
  const long long b = (tokens + (1 << a.block_shift) - 1) >> a.block_shift;
  return b < a.width ? b : a.width;
}
__device__ inline int plan_clamp(long long v) { return v > 0x7fffffffll ? 0x7fffffff : (int)v; }

__global__ void __launch_bounds__(PLAN_THREADS) k_kv_plan(PlanArgs a) {
  __shared__ int first_token[PLAN_SHARES], first_block[PLAN_SHARES];
  __shared__ long long wave_token[4], wave_block[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.shares + PLAN_THREADS - 1) / PLAN_THREADS * a.share;       // requests of a thread
  const long long r0 = (long long)tid * per;
  long long tokens = 0, blocks = 0;
#pragma unroll 4
  for (int k = 0; k < per; ++k) {
    const long long r = min(r0 + k, (long long)a.n - 1);
    const long long c = max(a.cached[r], 0), f = r0 + k < a.n ? max(a.fresh[r], 0) : 0;
    tokens += f;
    blocks += plan_blocks(c + f, a) - plan_blocks(c, a);
  }
  // inclusive sums over the wave, then over the waves
  long long t = tokens, b = blocks;
  for (int d = 1; d < 64; d <<= 1) {
    const long long pt = __shfl_up(t, d, 64), pb = __shfl_up(b, d, 64);
    if (lane >= d) { t += pt; b += pb; }
  }
  if (lane == 63) { wave_token[wave] = t; wave_block[wave] = b; }
  __syncthreads();
  long long total = 0, all_blocks = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) { t += wave_token[w]; b += wave_block[w]; }
    total += wave_token[w];
    all_blocks += wave_block[w];
  }
  t -= tokens;
  b -= blocks;
#pragma unroll 4
  for (int k = 0; k < per; ++k) {
    const long long r = r0 + k;
    if (r >= a.n) break;
    if (k % a.share == 0) {
      first_token[r / a.share] = plan_clamp(t);
      first_block[r / a.share] = plan_clamp(b);
    }
    const long long c = max(a.cached[r], 0), f = max(a.fresh[r], 0);
    if (blockIdx.x == 0) {
      a.starts[r] = plan_clamp(t);
      a.lengths[r] = plan_clamp(c + f);
    }
    t += f;
    b += plan_blocks(c + f, a) - plan_blocks(c, a);
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.starts[a.n] = plan_clamp(total);
    a.taken[0] = plan_clamp(all_blocks);
  }
  __syncthreads();

  const int i0 = (blockIdx.x * PLAN_THREADS + tid) * PLAN_TOKENS;
  // the last share that starts at or before the first token (shares without tokens in between are passed over: they start there
  // too)
  int lo = 0, hi = a.shares;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_token[mid] <= i0) lo = mid; else hi = mid;
  }
  long long r = (long long)lo * a.share, s = first_token[lo], nb = first_block[lo];
  long long c = max(a.cached[r], 0), f = max(a.fresh[r], 0);
#pragma unroll
  for (int k = 0; k < PLAN_TOKENS; ++k) {
    const int i = i0 + k;
    if (i >= a.max_tokens) break;
    int slot = -1, position = -1;
    if (i < total) {
      while (i >= s + f) {                                     // ends: token i is some request's
        s += f;
        nb += plan_blocks(c + f, a) - plan_blocks(c, a);
        ++r;
        c = max(a.cached[r], 0);
        f = max(a.fresh[r], 0);
      }
      const long long p = c + (i - s), pb = p >> a.block_shift;
      position = plan_clamp(p);
      if (pb < a.width) {
        const long long had = plan_blocks(c, a);
        int id;
        if (pb < had) id = a.table[r * a.width + pb];
        else {
          const long long at = nb + pb - had;
          id = at < a.n_free ? a.free_blocks[at] : -1;
          if ((p & ((1 << a.block_shift) - 1)) == 0) a.table[r * a.width + pb] = id;       // its block's first token
        }
        const long long v = ((long long)id << a.block_shift) + (p & ((1 << a.block_shift) - 1));
        if (id >= 0 && v <= 0x7fffffffll) slot = (int)v;
      }
    }
    a.slots[i] = slot;
    a.positions[i] = position;
  }
}

hipError_t launch_kv_plan(const glowq_kv_step& s, hipStream_t st) {
  const int share = (s.n_requests + PLAN_SHARES - 1) / PLAN_SHARES, shares = (s.n_requests + share - 1) / share;
  const PlanArgs a = {s.cached, s.fresh, s.free_blocks, s.table, s.lengths, s.starts, s.slots, s.positions, s.taken,
                      s.n_requests, s.n_free, s.table_width, s.max_tokens, kv_shift(s.block_tokens), share, shares};
  const int grid = (s.max_tokens + PLAN_THREADS * PLAN_TOKENS - 1) / (PLAN_THREADS * PLAN_TOKENS);
  k_kv_plan<<<dim3(grid), dim3(PLAN_THREADS), 0, st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// New tokens into the cache: the run's largest magnitude, the block's exponent, the codes.  Bytes in and out are the bound for
// prompts, the chain slot -> rows -> codes for single tokens.  Values are stored with the token as the fastest index: their
// codes pass through an image of the tiles in LDS and leave it in whole pieces; behind the run's last token a tile is filled
// with zeros.
struct AppendArgs {
  KvView cache;
  const uint16_t* rows[2];
  long long ld[2];
  const int32_t* slots;
  int T, per;
};

// TOKENS: of a run that a wave holds at once, whole 16-token tiles; 32 where blocks have no more, for more waves to a SIMD
template <int ACT, int DP, int TOKENS>
__global__ void __launch_bounds__(RUN_THREADS) k_kv_append(AppendArgs a) {
  __shared__ u32x4_t image_lds[RUN_WAVES / 2][TOKENS * DP * 4];                  // (every other wave has values)
  const int wave = threadIdx.x >> 6, pair = __builtin_amdgcn_readfirstlane(blockIdx.y * RUN_WAVES + wave);
  if (pair >= 2 * a.cache.kv_heads) return;
  const int which = pair & 1, head = pair >> 1;
  const uint16_t* const src = a.rows[which] + (size_t)head * 64 * DP;
  kv_runs(a.cache, a.slots, a.T, a.per, [&](int first, int slot, int m) {
    kv_append_run<ACT, DP, TOKENS>(a.cache, which, head, src, a.ld[which], image_lds[wave >> 1], first, slot, m);
  }, [](int) {});
}

hipError_t launch_kv_append(const glowq_kv_cache& cache, const void* k, int ldk, const void* v, int ldv, int act, const int32_t* slots,
                            int T, hipStream_t st) {
  const AppendArgs a = {kv_view(cache), {(const uint16_t*)k, (const uint16_t*)v}, {ldk, ldv}, slots, T, rows_per_wave(T, cache.kv_heads)};
  const dim3 grid((T + a.per - 1) / a.per, (2 * cache.kv_heads + RUN_WAVES - 1) / RUN_WAVES), block(RUN_THREADS);
#define GLOWQ_APPEND(DP, TOKENS) \
  act == GLOWQ_F16 ? k_kv_append<ACT_F16, DP, TOKENS><<<grid, block, 0, st>>>(a) : k_kv_append<ACT_BF16, DP, TOKENS><<<grid, block, 0, st>>>(a)
  if (cache.head_dim == 64) cache.block_tokens <= 32 ? (GLOWQ_APPEND(1, 32)) : (GLOWQ_APPEND(1, 64));
  else cache.block_tokens <= 32 ? (GLOWQ_APPEND(2, 32)) : (GLOWQ_APPEND(2, 64));
#undef GLOWQ_APPEND
  return hipGetLastError();
}

// Tokens back from the cache as numbers, run by run: keys straight from their pieces, values through an image of the tiles in LDS.
struct GatherArgs {
  KvView cache;
  void* rows[2];
  long long ld[2];
  const int32_t* slots;
  int T, per;
};

template <int TYPE, int DP>
__global__ void __launch_bounds__(RUN_THREADS) k_kv_gather(GatherArgs a) {
  constexpr int D = 64 * DP, PER_ROW = D / 16, TILE = 16 * D, TOKENS = 64, SIZE = TYPE == GLOWQ_F32 ? 4 : 2;
  __shared__ u32x4_t image_lds[RUN_WAVES / 2][TOKENS / 16 * TILE / 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pair = __builtin_amdgcn_readfirstlane(blockIdx.y * RUN_WAVES + wave);
  const KvView& c = a.cache;
  if (pair >= 2 * c.kv_heads) return;
  const int which = pair & 1, head = pair >> 1, B = 1 << c.block_shift;
  u32x4_t* const image = image_lds[wave >> 1];
  const int d = lane % PER_ROW * 16, token = lane / PER_ROW;
  const auto out = [&](int row) { return (u32x4_t*)((uint8_t*)a.rows[which] + ((size_t)row * a.ld[which] + (size_t)head * D + d) * SIZE); };
  kv_runs(c, a.slots, a.T, a.per, [&](int first, int slot, int m) {
    const int block = slot >> c.block_shift, off = slot & (B - 1), end = off + m;
    const uint8_t* const page = c.codes[which] + c.page(block, head);
    const float scale = kv_pow2((int)c.scales[which][(size_t)block * c.kv_heads + head] - 127);
    for (int from = off; from < end; ) {
      const int to = min(end, (from & ~15) + TOKENS), tile = from >> 4;
      if (which) {
        kv_wave_sync();
        constexpr int LOADS = TOKENS / 16 * TILE / 16 / 64;
        const int last = ((to + 15 >> 4) - tile) * (TILE / 16) - 1;
        u32x4_t w[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; ++k) w[k] = ((const u32x4_t*)page)[tile * (TILE / 16) + min(lane + 64 * k, last)];
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
          if (lane + 64 * k <= last) image[lane + 64 * k] = w[k];
        kv_wave_sync();
      }
#pragma unroll 4
      for (int t = from + token; t < to; t += 64 / PER_ROW) {
        u32x4_t w = {0, 0, 0, 0};
        if (!which) w = *(const u32x4_t*)(page + kv_key_byte(t, d, 6 + (DP == 2)));
        else {
          const uint8_t* const b = (const uint8_t*)image + kv_value_byte(t - tile * 16, d, 6 + (DP == 2));
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i >> 2] |= (uint32_t)b[16 * i] << (8 * (i & 3));
        }
        float x[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], true);
          x[4 * q] = lo[0] * scale; x[4 * q + 1] = lo[1] * scale; x[4 * q + 2] = hi[0] * scale; x[4 * q + 3] = hi[1] * scale;
        }
        u32x4_t* const to_row = out(first + t - off);
        if constexpr (TYPE == GLOWQ_F32) {
#pragma unroll
          for (int q = 0; q < 4; ++q) to_row[q] = __builtin_bit_cast(u32x4_t, float4_t{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]});
        } else {
          u32x4_t o[2];
#pragma unroll
          for (int q = 0; q < 8; ++q)
            o[q >> 2][q & 3] = (uint32_t)to_act16<TYPE == GLOWQ_F16 ? ACT_F16 : ACT_BF16>(x[2 * q]) |
                               (uint32_t)to_act16<TYPE == GLOWQ_F16 ? ACT_F16 : ACT_BF16>(x[2 * q + 1]) << 16;
          to_row[0] = o[0];
          to_row[1] = o[1];
        }
      }
      from = to;
    }
  }, [&](int row) {
    if (lane < PER_ROW)
#pragma unroll
      for (int q = 0; q < SIZE; ++q) out(row)[q] = u32x4_t{0, 0, 0, 0};
  });
}

template <int DP> static void gather(const GatherArgs& a, int dtype, dim3 grid, hipStream_t st) {
  if (dtype == GLOWQ_F16) k_kv_gather<GLOWQ_F16, DP><<<grid, dim3(RUN_THREADS), 0, st>>>(a);
  else if (dtype == GLOWQ_BF16) k_kv_gather<GLOWQ_BF16, DP><<<grid, dim3(RUN_THREADS), 0, st>>>(a);
  else k_kv_gather<GLOWQ_F32, DP><<<grid, dim3(RUN_THREADS), 0, st>>>(a);
}
hipError_t launch_kv_gather(const glowq_kv_cache& cache, const int32_t* slots, int T, void* k, int ldk, void* v, int ldv, int dtype,
                            hipStream_t st) {
  const GatherArgs a = {kv_view(cache), {k, v}, {ldk, ldv}, slots, T, rows_per_wave(T, cache.kv_heads)};
  const dim3 grid((T + a.per - 1) / a.per, (2 * cache.kv_heads + RUN_WAVES - 1) / RUN_WAVES);
  cache.head_dim == 64 ? gather<1>(a, dtype, grid, st) : gather<2>(a, dtype, grid, st);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// Argument checks
static bool bad16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
static bool bad4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

static glowq_status check_block_tokens(int b) { return b == 16 || b == 32 || b == 64 || b == 128 ? GLOWQ_OK : b < 1 ? GLOWQ_ERR_SHAPE : GLOWQ_ERR_UNSUPPORTED; }

// sizes first; what is well formed but not served afterwards
glowq_status kv_check_cache(const glowq_kv_cache* c, bool ptrs) {
  if (!c) return GLOWQ_ERR_NULL;
  if (c->n_blocks < 1 || c->kv_heads < 1 || c->kv_heads > 1024 || c->head_dim < 1) return GLOWQ_ERR_SHAPE;
  glowq_status s = check_block_tokens(c->block_tokens);
  if (s != GLOWQ_OK) return s;
  if (c->head_dim != 64 && c->head_dim != 128) return GLOWQ_ERR_UNSUPPORTED;
  if ((long long)c->n_blocks * c->block_tokens > 0x7fffffffll) return GLOWQ_ERR_SHAPE;         // slots are 32-bit
  if (!ptrs) return GLOWQ_OK;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return GLOWQ_ERR_NULL;
  return bad16(c->k_codes) || bad16(c->v_codes) || bad16(c->k_scales) || bad16(c->v_scales) ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

glowq_status kv_check_rows(const glowq_kv_cache* c, const void* k, int ldk, const void* v, int ldv, const int32_t* slots, int T) {
  glowq_status s = kv_check_cache(c, true);
  if (s != GLOWQ_OK) return s;
  if (T < 1 || T > (1 << 20)) return GLOWQ_ERR_SHAPE;
  const int w = c->kv_heads * c->head_dim;
  if (ldk < w || ldv < w) return GLOWQ_ERR_SHAPE;
  if (ldk % 8 || ldv % 8) return GLOWQ_ERR_UNSUPPORTED;
  if (!k || !v || !slots) return GLOWQ_ERR_NULL;
  return bad16(k) || bad16(v) || bad4(slots) ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

}  // namespace glowq

using namespace glowq;
extern "C" {

glowq_status glowq_kv_cache_bytes(const glowq_kv_cache* cache, size_t* code_bytes, size_t* scale_bytes) {
  if (!code_bytes || !scale_bytes) return GLOWQ_ERR_NULL;
  const glowq_status s = kv_check_cache(cache, false);
  if (s != GLOWQ_OK) return s;
  *scale_bytes = (size_t)cache->n_blocks * cache->kv_heads;
  *code_bytes = *scale_bytes * cache->block_tokens * cache->head_dim;
  return GLOWQ_OK;
}

glowq_status glowq_kv_plan(const glowq_kv_step* p, void* stream) {
  if (!p) return GLOWQ_ERR_NULL;
  if (p->n_requests < 1 || p->n_requests > (1 << 20) || p->n_free < 0 || p->table_width < 1 || p->max_tokens < 1 || p->max_tokens > (1 << 20))
    return GLOWQ_ERR_SHAPE;
  const glowq_status s = check_block_tokens(p->block_tokens);
  if (s != GLOWQ_OK) return s;
  if (!p->cached || !p->fresh || (!p->free_blocks && p->n_free > 0) || !p->table || !p->lengths || !p->starts || !p->slots || !p->positions || !p->taken)
    return GLOWQ_ERR_NULL;
  for (const void* q : {(const void*)p->cached, (const void*)p->fresh, (const void*)p->free_blocks, (const void*)p->table, (const void*)p->lengths,
                        (const void*)p->starts, (const void*)p->slots, (const void*)p->positions, (const void*)p->taken})
    if (bad4(q)) return GLOWQ_ERR_ALIGN;
  return hip_status(launch_kv_plan(*p, (hipStream_t)stream));
}

glowq_status glowq_kv_append(const glowq_kv_cache* cache, const void* k, int32_t ldk, const void* v, int32_t ldv, int32_t act_dtype,
                             const int32_t* slots, int32_t T, void* stream) {
  const glowq_status s = kv_check_rows(cache, k, ldk, v, ldv, slots, T);
  if (s != GLOWQ_OK) return s;
  if (act_dtype != GLOWQ_F16 && act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  return hip_status(launch_kv_append(*cache, k, ldk, v, ldv, act_dtype, slots, T, (hipStream_t)stream));
}

glowq_status glowq_kv_gather(const glowq_kv_cache* cache, const int32_t* slots, int32_t T, void* k, int32_t ldk, void* v, int32_t ldv,
                             int32_t dtype, void* stream) {
  const glowq_status s = kv_check_rows(cache, k, ldk, v, ldv, slots, T);
  if (s != GLOWQ_OK) return s;
  if (dtype != GLOWQ_F16 && dtype != GLOWQ_BF16 && dtype != GLOWQ_F32) return GLOWQ_ERR_DTYPE;
  return hip_status(launch_kv_gather(*cache, slots, T, k, ldk, v, ldv, dtype, (hipStream_t)stream));
}

}  // extern "C"
