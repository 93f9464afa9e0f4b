// The 8-bit cache of keys and values: block tables and slot maps of a step, new tokens into the cache, tokens read back.
#include <algorithm>
#include "kv_device.hpp"
#include "kv_host.hpp"

namespace glowq {

// ---------------------------------------------------------------------------------------
// Tables and slots of a step.  Two running sums over the requests (tokens, blocks) and one look-up per token; the work is
// a few bytes per token, so the launch and its chain of dependent loads are the time.  Every workgroup adds up all requests
// itself (8 bytes each, from the L2 after the first) rather than waiting for one that does: one launch, nothing to hand over.
// Thread i of a workgroup sums `per` consecutive requests; a token finds its thread's share by bisection in LDS and walks
// within it.
constexpr int PLAN_THREADS = 256;
constexpr int PLAN_TOKENS = 1024;      // per workgroup

struct PlanArgs {
  const int32_t *cached, *fresh, *free_blocks;
  int32_t *table, *lengths, *starts, *slots, *positions, *taken;
  int n, n_free, width, max_tokens, block_shift, per;
};

__device__ inline long long plan_blocks(long long tokens, const PlanArgs& a) {
  const long long b = (tokens + (1 << a.block_shift) - 1) >> a.block_shift;
  return b < a.width ? b : a.width;
}
__device__ inline int plan_clamp(long long v) { return v > 0x7fffffffll ? 0x7fffffff : (int)v; }

__global__ void __launch_bounds__(PLAN_THREADS) k_kv_plan(PlanArgs a) {
  __shared__ long long first_token[PLAN_THREADS + 1], first_block[PLAN_THREADS + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long r0 = (long long)tid * a.per;
  long long tokens = 0, blocks = 0;
  for (int k = 0; k < a.per && r0 + k < a.n; ++k) {
    const long long c = max(a.cached[r0 + k], 0), f = max(a.fresh[r0 + k], 0);
    tokens += f;
    blocks += plan_blocks(c + f, a) - plan_blocks(c, a);
  }
  // inclusive sums over the wave, then over the waves
  long long t = tokens, b = blocks;
  for (int d = 1; d < 64; d <<= 1) {
    const long long pt = __shfl_up(t, d, 64), pb = __shfl_up(b, d, 64);
    if (lane >= d) { t += pt; b += pb; }
  }
  __shared__ long long wave_token[4], wave_block[4];
  if (lane == 63) { wave_token[wave] = t; wave_block[wave] = b; }
  __syncthreads();
  for (int w = 0; w < wave; ++w) { t += wave_token[w]; b += wave_block[w]; }
  first_token[tid] = t - tokens;
  first_block[tid] = b - blocks;
  if (tid == PLAN_THREADS - 1) { first_token[PLAN_THREADS] = t; first_block[PLAN_THREADS] = b; }
  __syncthreads();

  if (blockIdx.x == 0) {
    long long s = first_token[tid];
    for (int k = 0; k < a.per && r0 + k < a.n; ++k) {
      const long long c = max(a.cached[r0 + k], 0), f = max(a.fresh[r0 + k], 0);
      a.starts[r0 + k] = plan_clamp(s);
      a.lengths[r0 + k] = plan_clamp(c + f);
      s += f;
    }
    if (tid == 0) {
      a.starts[a.n] = plan_clamp(first_token[PLAN_THREADS]);
      a.taken[0] = plan_clamp(first_block[PLAN_THREADS]);
    }
  }
  const long long total = first_token[PLAN_THREADS];
  for (int k = 0; k < PLAN_TOKENS / PLAN_THREADS; ++k) {
    const long long i = (long long)blockIdx.x * PLAN_TOKENS + k * PLAN_THREADS + tid;
    if (i >= a.max_tokens) break;
    int slot = -1, position = -1;
    if (i < total) {
      // the last share that starts at or before i (shares without tokens in between are passed over: they start there too)
      int lo = 0, hi = PLAN_THREADS;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_token[mid] <= i) lo = mid; else hi = mid;
      }
      long long r = (long long)lo * a.per, s = first_token[lo], nb = first_block[lo], c = 0;
      for (;; ++r) {                                           // ends: the share holds token i
        c = max(a.cached[r], 0);
        const long long f = max(a.fresh[r], 0);
        if (i < s + f) break;
        s += f;
        nb += plan_blocks(c + f, a) - plan_blocks(c, a);
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
  PlanArgs a = {s.cached, s.fresh, s.free_blocks, s.table, s.lengths, s.starts, s.slots, s.positions, s.taken,
                s.n_requests, s.n_free, s.table_width, s.max_tokens, kv_shift(s.block_tokens),
                (s.n_requests + PLAN_THREADS - 1) / PLAN_THREADS};
  const int grid = std::max(1, (s.max_tokens + PLAN_TOKENS - 1) / PLAN_TOKENS);
  k_kv_plan<<<dim3(grid), dim3(PLAN_THREADS), 0, st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// New tokens into the cache.  A run is a stretch of rows whose slots follow each other within one block; one workgroup takes
// the runs that begin in its rows, one after another, for one head's keys or values: the run's largest magnitude, the
// block's exponent, the codes.  Bytes in and out are the bound for prompts, the chain slot -> rows -> codes for single
// tokens.  Values are stored with the token as the fastest index, so their codes pass through an image of the page in LDS and
// leave it as whole words of four tokens; behind the run's last token the word is filled with zeros.
constexpr int APPEND_THREADS = 256;

struct AppendArgs {
  KvView cache;
  const uint16_t* rows[2];
  long long ld[2];
  const int32_t* slots;
  int T, per;              // rows; rows per workgroup
};

template <int ACT>
__global__ void __launch_bounds__(APPEND_THREADS) k_kv_append(AppendArgs a) {
  __shared__ uint32_t page_lds[128 * 128 / 4];       // the touched tiles of a page of values
  __shared__ uint32_t wave_top[APPEND_THREADS / 64];
  __shared__ int run_end;
  const int tid = threadIdx.x, which = blockIdx.y & 1, head = blockIdx.y >> 1;
  const KvView& c = a.cache;
  const int B = 1 << c.block_shift, D = 1 << c.dim_shift, per_row = D / 16;
  const uint16_t* const src = a.rows[which] + (size_t)head * D;
  const int row_end = min(a.T, (int)(blockIdx.x + 1) * a.per);
  int row = blockIdx.x * a.per;
  while (row < row_end) {
    const int s0 = a.slots[row];
    const int block = s0 >> c.block_shift, off = s0 & (B - 1);
    const bool valid = s0 >= 0 && block < c.n_blocks;
    // a row that goes on from the one before it belongs to that one's run
    if (!valid || (row > 0 && off > 0 && a.slots[row - 1] == s0 - 1)) { ++row; continue; }
    __syncthreads();                                 // the run before is done with the shared words
    if (tid == 0) run_end = min(B - off, a.T - row);
    __syncthreads();
    if (tid < min(B - off, a.T - row) && a.slots[row + tid] != s0 + tid) atomicMin(&run_end, tid);
    __syncthreads();
    const int m = run_end;

    // the run's largest finite magnitude, by its bits
    uint32_t top = 0;
    for (int u = tid; u < m * per_row; u += APPEND_THREADS) {
      const u32x4_t* p = (const u32x4_t*)(src + (size_t)(row + u / per_row) * a.ld[which] + (u % per_row) * 16);
      const u32x4_t x[2] = {p[0], p[1]};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t w = x[i >> 2][i & 3];
        const uint32_t lo = __builtin_bit_cast(uint32_t, kv_act_f32<ACT>(w & 0x7fffu)), hi = __builtin_bit_cast(uint32_t, kv_act_f32<ACT>((w >> 16) & 0x7fffu));
        if (lo < 0x7f800000u) top = max(top, lo);
        if (hi < 0x7f800000u) top = max(top, hi);
      }
    }
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
    for (int w = 0; w < APPEND_THREADS / 64; ++w) top = max(top, wave_top[w]);

    uint8_t* const scale = c.scales[which] + (size_t)block * c.kv_heads + head;
    uint8_t* const page = c.codes[which] + c.page(block, head);
    const int before = off > 0 ? min((int)*scale - 127, 126) : KV_EXP_MIN;
    const int e = max(before, kv_exponent(top));
    const float inv = kv_pow2(-e), shrink = kv_pow2(max(before - e, -126));
    const bool grown = off > 0 && e > before;
    __syncthreads();                                 // everyone has the old scale
    if (tid == 0 && (off == 0 || grown)) *scale = (uint8_t)(e + 127);

    const int pieces = D / 64;
    const int tile0 = off >> 4, tile1 = (off + m - 1) >> 4;            // tiles that the run touches
    if (which == 0) {
      if (grown)                                     // older tokens of the block to the new grid
        for (int u = tid; u < ((off + 15) >> 4) * pieces * 64; u += APPEND_THREADS) {
          if ((u / (pieces * 64)) * 16 + (u & 15) >= off) continue;
          u32x4_t* p = (u32x4_t*)page + u;
          u32x4_t w = *p;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = kv_recode4(w[i], shrink);
          *p = w;
        }
    } else {
      const int from = grown ? 0 : tile0;            // tiles from here on go through LDS
      const int words = (tile1 + 1 - from) * pieces * (KV_PIECE / 4);
      for (int u = tid; u < words; u += APPEND_THREADS) {
        const int at = u + from * pieces * (KV_PIECE / 4);
        const int t0 = at / (pieces * 256) * 16 + ((at >> 6) & 3) * 4;     // first of the word's four tokens
        uint32_t w = 0;
        if (t0 < off) {
          w = ((const uint32_t*)page)[at];
          if (grown) w = kv_recode4(w, shrink);
          if (t0 + 4 > off) w &= 0xffffffffu >> (8 * (t0 + 4 - off));
        }
        page_lds[u] = w;
      }
      __syncthreads();
    }
    for (int u = tid; u < m * per_row; u += APPEND_THREADS) {
      const int i = u / per_row, d = (u % per_row) * 16, t = off + i;
      const u32x4_t* p = (const u32x4_t*)(src + (size_t)(row + i) * a.ld[which] + d);
      const u32x4_t x[2] = {p[0], p[1]};
      u32x4_t code;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t w0 = x[q >> 1][(q & 1) * 2], w1 = x[q >> 1][(q & 1) * 2 + 1];
        code[q] = kv_encode4(kv_act_f32<ACT>(w0 & 0xffffu) * inv, kv_act_f32<ACT>(w0 >> 16) * inv, kv_act_f32<ACT>(w1 & 0xffffu) * inv,
                             kv_act_f32<ACT>(w1 >> 16) * inv);
      }
      if (which == 0) *(u32x4_t*)(page + kv_key_byte(t, d, c.dim_shift)) = code;
      else {
        uint8_t* const b = (uint8_t*)page_lds + kv_value_byte(t, d, c.dim_shift) - (grown ? 0 : tile0) * pieces * KV_PIECE;
#pragma unroll
        for (int k = 0; k < 16; ++k) b[16 * k] = (uint8_t)(code[k >> 2] >> (8 * (k & 3)));
      }
    }
    if (which == 1) {
      __syncthreads();
      const int from = grown ? 0 : tile0, chunks = (tile1 + 1 - from) * pieces * 64;
      for (int u = tid; u < chunks; u += APPEND_THREADS) ((u32x4_t*)page)[u + from * pieces * 64] = ((const u32x4_t*)page_lds)[u];
    }
    row += m;
  }
}

hipError_t launch_kv_append(const glowq_kv_cache& cache, const void* k, int ldk, const void* v, int ldv, int act, const int32_t* slots,
                            int T, hipStream_t st) {
  AppendArgs a = {kv_view(cache), {(const uint16_t*)k, (const uint16_t*)v}, {ldk, ldv}, slots, T, 1};
  a.per = (long long)T * cache.kv_heads <= 8192 ? 1 : 16;
  const dim3 grid((T + a.per - 1) / a.per, 2 * cache.kv_heads);
  if (act == GLOWQ_F16) k_kv_append<ACT_F16><<<grid, dim3(APPEND_THREADS), 0, st>>>(a);
  else k_kv_append<ACT_BF16><<<grid, dim3(APPEND_THREADS), 0, st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// Tokens back from the cache as numbers: one thread per 16 dims of a token's keys or values.
struct GatherArgs {
  KvView cache;
  void* rows[2];
  long long ld[2];
  const int32_t* slots;
  int T;
};

template <int TYPE>
__global__ void __launch_bounds__(256) k_kv_gather(GatherArgs a) {
  const KvView& c = a.cache;
  const int B = 1 << c.block_shift, D = 1 << c.dim_shift;
  const int units = c.kv_heads * D / 16;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long row = at / units;
  if (row >= a.T) return;
  const int u = (int)(at - row * units), which = blockIdx.y, head = u / (D / 16), d = u % (D / 16) * 16;
  const int slot = a.slots[row], block = slot >> c.block_shift;
  u32x4_t w = {0, 0, 0, 0};
  float scale = 0.f;
  if (slot >= 0 && block < c.n_blocks) {
    const uint8_t* page = c.codes[which] + c.page(block, head);
    if (which == 0) w = *(const u32x4_t*)(page + kv_key_byte(slot & (B - 1), d, c.dim_shift));
    else {
      const uint8_t* p = page + kv_value_byte(slot & (B - 1), d, c.dim_shift);
#pragma unroll
      for (int k = 0; k < 16; ++k) w[k >> 2] |= (uint32_t)p[16 * k] << (8 * (k & 3));
    }
    scale = kv_pow2((int)c.scales[which][(size_t)block * c.kv_heads + head] - 127);
  }
  float x[16];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[q], true);
    x[4 * q] = lo[0] * scale; x[4 * q + 1] = lo[1] * scale; x[4 * q + 2] = hi[0] * scale; x[4 * q + 3] = hi[1] * scale;
  }
  const size_t to = (size_t)row * a.ld[which] + (size_t)head * D + d;
  if constexpr (TYPE == GLOWQ_F32) {
    float4_t* p = (float4_t*)((float*)a.rows[which] + to);
#pragma unroll
    for (int q = 0; q < 4; ++q) p[q] = float4_t{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
  } else {
    u32x4_t o[2];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      o[q >> 2][q & 3] = (uint32_t)to_act16<TYPE == GLOWQ_F16 ? ACT_F16 : ACT_BF16>(x[2 * q]) |
                         (uint32_t)to_act16<TYPE == GLOWQ_F16 ? ACT_F16 : ACT_BF16>(x[2 * q + 1]) << 16;
    u32x4_t* p = (u32x4_t*)((uint16_t*)a.rows[which] + to);
    p[0] = o[0];
    p[1] = o[1];
  }
}

hipError_t launch_kv_gather(const glowq_kv_cache& cache, const int32_t* slots, int T, void* k, int ldk, void* v, int ldv, int dtype,
                            hipStream_t st) {
  const GatherArgs a = {kv_view(cache), {k, v}, {ldk, ldv}, slots, T};
  const long long n = (long long)T * cache.kv_heads * cache.head_dim / 16;
  const dim3 grid((unsigned)((n + 255) / 256), 2);
  if (dtype == GLOWQ_F16) k_kv_gather<GLOWQ_F16><<<grid, dim3(256), 0, st>>>(a);
  else if (dtype == GLOWQ_BF16) k_kv_gather<GLOWQ_BF16><<<grid, dim3(256), 0, st>>>(a);
  else k_kv_gather<GLOWQ_F32><<<grid, dim3(256), 0, st>>>(a);
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

static glowq_status check_rows(const glowq_kv_cache* c, const void* k, int ldk, const void* v, int ldv, const int32_t* slots, int T) {
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
  const glowq_status s = check_rows(cache, k, ldk, v, ldv, slots, T);
  if (s != GLOWQ_OK) return s;
  if (act_dtype != GLOWQ_F16 && act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  return hip_status(launch_kv_append(*cache, k, ldk, v, ldv, act_dtype, slots, T, (hipStream_t)stream));
}

glowq_status glowq_kv_gather(const glowq_kv_cache* cache, const int32_t* slots, int32_t T, void* k, int32_t ldk, void* v, int32_t ldv,
                             int32_t dtype, void* stream) {
  const glowq_status s = check_rows(cache, k, ldk, v, ldv, slots, T);
  if (s != GLOWQ_OK) return s;
  if (dtype != GLOWQ_F16 && dtype != GLOWQ_BF16 && dtype != GLOWQ_F32) return GLOWQ_ERR_DTYPE;
  return hip_status(launch_kv_gather(*cache, slots, T, k, ldk, v, ldv, dtype, (hipStream_t)stream));
}

}  // extern "C"
