// The latent cache: new tokens into it, tokens read back; the per-head maps into and out of the latents.
#include <algorithm>
#include "latent_host.hpp"
#include "rope_host.hpp"

namespace glowq {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------------------
// New tokens.  A wave a token: the latent's largest magnitude by shuffles, its exponent, its codes; the key part rotated by the
// first lanes.  Behind them workgroups that rotate q.  Bytes are the bound for prompts, the launch and its chain for single tokens.
constexpr int LATENT_THREADS = 256, LATENT_WAVES = LATENT_THREADS / 64;

struct LatentAppendArgs {
  LatentView cache;
  const uint16_t *c, *r;
  long long ldc, ldr;
  const int32_t *slots, *positions;
  RopeView rope;               // units 0: the key parts as they stand
  RotateArgs q;
  int T, cache_blocks, rope_units;
};

template <int ACT, int LATENT>
__global__ void __launch_bounds__(LATENT_THREADS) k_latent_append(LatentAppendArgs a) {
  constexpr int PER = LATENT / 64, WORDS = PER / 2;
  constexpr uint32_t INF = ACT == ACT_F16 ? 0x7c00u : 0x7f80u;
  if ((int)blockIdx.x >= a.cache_blocks) {
    rope_rotate<ACT>(a.q, (long long)(blockIdx.x - a.cache_blocks) * LATENT_THREADS + threadIdx.x);
    return;
  }
  const int lane = threadIdx.x & 63, row = blockIdx.x * LATENT_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.T) return;
  const int slot = __builtin_amdgcn_readfirstlane(a.slots[row]);
  const uint16_t* const src = a.c + row * a.ldc + PER * lane;
  uint32_t w[WORDS];
#pragma unroll
  for (int i = 0; i < WORDS; i += 2) {
    const u32x2_t v = *(const u32x2_t*)(src + 2 * i);
    w[i] = v[0];
    w[i + 1] = v[1];
  }
  if (!a.cache.has(slot)) return;
  if (lane < a.rope_units) {
    RopeView rope = a.rope;
    const bool turn = rope.units > 0;
    if (!turn) rope.pairs = 1;             // (16 dims as they stand)
    const int da = rope.dim_a(lane), db = rope.dim_b(lane);
    float u[8], v[8];
    rope_load16<ACT>(a.r + row * a.ldr + da, u);
    rope_load16<ACT>(a.r + row * a.ldr + db, v);
    if (turn && lane < rope.units) {
      RopeAngles<8> angle;
      angle.set(rope, 8 * lane, max(a.positions[row], 0));
      rope_turn_unit(u, v, angle.c, angle.s, rope.pairs);
    }
    uint16_t* const to = a.cache.ropes + (size_t)slot * 16 * a.rope_units;
    rope_store16<ACT>(to + da, u);
    rope_store16<ACT>(to + db, v);
  }
  // the largest finite magnitude, by its bits
  uint32_t h = 0;
#pragma unroll
  for (int i = 0; i < WORDS; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = w[i] >> 16 & 0x7fffu;
    h = lo < INF ? max(h, lo) : h;
    h = hi < INF ? max(h, hi) : h;
  }
  for (int k = 1; k < 64; k <<= 1) h = max(h, (uint32_t)__shfl_xor((int)h, k, 64));
  const int e = max(kv_exponent(__builtin_bit_cast(uint32_t, kv_act_f32<ACT>(h))), LatentRange<ACT>::LOW);
  // (MOST is in reach at the type's largest exponent only; below it `most` passes 448)
  const float down = kv_pow2(-e), most = LatentRange<ACT>::MOST * down;
  uint32_t code[WORDS / 2];
#pragma unroll
  for (int i = 0; i < WORDS; i += 2) {
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = kv_act_f32<ACT>(w[i + (k >> 1)] >> (16 * (k & 1)) & 0xffffu) * down;
      // (what is not finite passes through to the NaN code)
      if (__builtin_fabsf(x[k]) < INFINITY) x[k] = __builtin_fminf(__builtin_fmaxf(x[k], -most), most);
    }
    code[i / 2] = kv_encode4(x[0], x[1], x[2], x[3]);
  }
  uint8_t* const to = a.cache.codes + (size_t)slot * LATENT + PER * lane;
  if constexpr (PER == 8) *(u32x2_t*)to = u32x2_t{code[0], code[1]};
  else *(uint32_t*)to = code[0];
  if (lane == 0) a.cache.scales[slot] = (uint8_t)(e + 127);
}

static hipError_t launch_latent_append(const glowq_latent_cache& cache, const glowq_rope* rope, const glowq_rope_rows* q, const void* c, int ldc,
                                       const void* r, int ldr, const int32_t* slots, const int32_t* positions, int T, hipStream_t st) {
  LatentAppendArgs a = {};
  a.cache = latent_view(cache);
  a.c = (const uint16_t*)c;
  a.r = (const uint16_t*)r;
  a.ldc = ldc;
  a.ldr = ldr;
  a.slots = slots;
  a.positions = positions;
  if (rope) a.rope = rope_view(*rope);
  a.T = T;
  a.rope_units = cache.rope_dim / 16;
  a.cache_blocks = (T + LATENT_WAVES - 1) / LATENT_WAVES;
  long long threads = 0;
  if (q) a.q = make_rotate_args(*rope, q, 1, cache.rope_dim, cache.act_dtype, positions, T, &threads);
  const dim3 grid((unsigned)(a.cache_blocks + (threads + LATENT_THREADS - 1) / LATENT_THREADS)), block(LATENT_THREADS);
  if (cache.act_dtype == GLOWQ_F16) {
    if (cache.latent_dim == 512) k_latent_append<ACT_F16, 512><<<grid, block, 0, st>>>(a);
    else k_latent_append<ACT_F16, 256><<<grid, block, 0, st>>>(a);
  } else {
    if (cache.latent_dim == 512) k_latent_append<ACT_BF16, 512><<<grid, block, 0, st>>>(a);
    else k_latent_append<ACT_BF16, 256><<<grid, block, 0, st>>>(a);
  }
  return hipGetLastError();
}

// Tokens back from the cache, a wave each.  Codes times their scale are numbers of the cache's type.
struct LatentGatherArgs {
  LatentView cache;
  const int32_t* slots;
  uint16_t *c, *r;
  long long ldc, ldr;
  int T, rope_dim;
};

template <int ACT, int LATENT>
__global__ void __launch_bounds__(LATENT_THREADS) k_latent_gather(LatentGatherArgs a) {
  constexpr int PER = LATENT / 64;
  const int lane = threadIdx.x & 63, row = blockIdx.x * LATENT_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.T) return;
  const int slot = __builtin_amdgcn_readfirstlane(a.slots[row]);
  const bool there = a.cache.has(slot);
  const size_t from = there ? slot : 0;
  const float scale = there ? kv_pow2((int)a.cache.scales[from] - 127) : 0.f;
  uint32_t out[PER / 2];
#pragma unroll
  for (int i = 0; i < PER / 4; ++i) {
    const uint32_t w = there ? ((const uint32_t*)(a.cache.codes + from * LATENT + PER * lane))[i] : 0u;
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    out[2 * i] = (uint32_t)to_act16<ACT>(lo[0] * scale) | (uint32_t)to_act16<ACT>(lo[1] * scale) << 16;
    out[2 * i + 1] = (uint32_t)to_act16<ACT>(hi[0] * scale) | (uint32_t)to_act16<ACT>(hi[1] * scale) << 16;
  }
  uint16_t* const to = a.c + row * a.ldc + PER * lane;
  if constexpr (PER == 8) *(u32x4_t*)to = u32x4_t{out[0], out[1], out[2], out[3]};
  else *(u32x2_t*)to = u32x2_t{out[0], out[1]};
  if (8 * lane < a.rope_dim) {
    const u32x4_t zero = {0, 0, 0, 0};
    *(u32x4_t*)(a.r + row * a.ldr + 8 * lane) = there ? *(const u32x4_t*)(a.cache.ropes + from * a.rope_dim + 8 * lane) : zero;
  }
}

static hipError_t launch_latent_gather(const glowq_latent_cache& cache, const int32_t* slots, int T, void* c, int ldc, void* r, int ldr, hipStream_t st) {
  const LatentGatherArgs a = {latent_view(cache), slots, (uint16_t*)c, (uint16_t*)r, ldc, ldr, T, cache.rope_dim};
  const dim3 grid((T + LATENT_WAVES - 1) / LATENT_WAVES), block(LATENT_THREADS);
  if (cache.act_dtype == GLOWQ_F16) {
    if (cache.latent_dim == 512) k_latent_gather<ACT_F16, 512><<<grid, block, 0, st>>>(a);
    else k_latent_gather<ACT_F16, 256><<<grid, block, 0, st>>>(a);
  } else {
    if (cache.latent_dim == 512) k_latent_gather<ACT_BF16, 512><<<grid, block, 0, st>>>(a);
    else k_latent_gather<ACT_BF16, 256><<<grid, block, 0, st>>>(a);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// Per-head maps, Y_h = X_h W_h^T.  A wave takes 16 outputs of a head and tokens in blocks of 16 * TB: Y^T = W X^T, so that
// a lane ends with four outputs in a row of one token.  Operands come from memory as they lie there, eight channels a lane; the
// maps are read once for every 16 * TB tokens.  Bound: the maps' bytes for few tokens (64 heads, 512 to 128: 7 to 8 us up to 32 tokens, where 128
// workgroups leave half of the machine without any); for many the tokens, which come from the caches once for every 16 outputs (21, 39 and 149 us
// for 256, 512 and 2048; 1.2 TB/s, 0.11 PFLOP/s).
struct HeadMapArgs {
  const uint16_t *x, *w;
  uint16_t* y;
  long long ldx, lhx, ldy, lhy;
  int T, d_in, d_out, heads;
};

template <int ACT, int TB>
__global__ void __launch_bounds__(256) k_head_maps(HeadMapArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int tiles = a.d_out / 16, tile = blockIdx.x * 4 + wave;
  if (tile >= tiles * a.heads) return;
  const int head = tile / tiles, n0 = (tile - head * tiles) * 16, t0 = blockIdx.y * 16 * TB;
  const uint16_t* const w = a.w + ((size_t)head * a.d_out + n0 + c) * a.d_in + 8 * g;
  const uint16_t* x[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) x[b] = a.x + min(t0 + 16 * b + c, a.T - 1) * a.ldx + head * a.lhx + 8 * g;
  float4_t sum[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) sum[b] = float4_t{0.f, 0.f, 0.f, 0.f};
  // stretches of N times 32 channels, one on its way while another is multiplied
  constexpr int N = TB == 4 ? 4 : 8;
  u32x4_t wk[2][N], xk[2][N][TB];
  const auto load = [&](int k, int to, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i >= n) continue;
      wk[to][i] = *(const u32x4_t*)(w + k + 32 * i);
#pragma unroll
      for (int b = 0; b < TB; ++b) xk[to][i][b] = *(const u32x4_t*)(x[b] + k + 32 * i);
    }
  };
  const auto multiply = [&](int from, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n)
#pragma unroll
        for (int b = 0; b < TB; ++b) sum[b] = mfma16<ACT>(wk[from][i], xk[from][i][b], sum[b]);
  };
  const int whole = a.d_in / (32 * N), rest = a.d_in / 32 % N;
  if (whole) load(0, 0, N);
  for (int s = 0; s < whole; s += 2) {
    if (s + 1 < whole) load(32 * N * (s + 1), 1, N);
    multiply(0, N);
    if (s + 1 < whole) {
      if (s + 2 < whole) load(32 * N * (s + 2), 0, N);
      multiply(1, N);
    }
  }
  if (rest) {
    load(32 * N * whole, 0, rest);
    multiply(0, rest);
  }
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int t = t0 + 16 * b + c;
    if (t >= a.T) continue;
    *(u32x2_t*)(a.y + t * a.ldy + head * a.lhy + n0 + 4 * g) =
        u32x2_t{(uint32_t)to_act16<ACT>(sum[b][0]) | (uint32_t)to_act16<ACT>(sum[b][1]) << 16, (uint32_t)to_act16<ACT>(sum[b][2]) | (uint32_t)to_act16<ACT>(sum[b][3]) << 16};
  }
}

template <int ACT> static void head_maps(const HeadMapArgs& a, hipStream_t st) {
  const unsigned tiles = (unsigned)((a.d_out / 16 * a.heads + 3) / 4);
  if (a.T <= 16) k_head_maps<ACT, 1><<<dim3(tiles, 1), dim3(256), 0, st>>>(a);
  else if (a.T <= 32) k_head_maps<ACT, 2><<<dim3(tiles, 1), dim3(256), 0, st>>>(a);
  else k_head_maps<ACT, 4><<<dim3(tiles, (a.T + 63) / 64), dim3(256), 0, st>>>(a);
}

// ---------------------------------------------------------------------------------------
// Argument checks
static bool bad16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
static bool bad4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

glowq_status latent_check_cache(const glowq_latent_cache* c, bool ptrs) {
  if (!c) return GLOWQ_ERR_NULL;
  if (c->n_blocks < 1 || c->latent_dim < 1 || c->rope_dim < 1 || c->block_tokens < 1) return GLOWQ_ERR_SHAPE;
  if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128) return GLOWQ_ERR_UNSUPPORTED;
  if ((c->latent_dim != 256 && c->latent_dim != 512) || (c->rope_dim != 32 && c->rope_dim != 64)) return GLOWQ_ERR_UNSUPPORTED;
  if ((long long)c->n_blocks * c->block_tokens > 0x7fffffffll) return GLOWQ_ERR_SHAPE;         // slots are 32-bit
  if (c->act_dtype != GLOWQ_F16 && c->act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  if (!ptrs) return GLOWQ_OK;
  if (!c->codes || !c->scales || !c->ropes) return GLOWQ_ERR_NULL;
  return bad16(c->codes) || bad16(c->scales) || bad16(c->ropes) ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

static glowq_status check_rows(const glowq_latent_cache* cache, const void* c, int ldc, const void* r, int ldr, const int32_t* slots, int T) {
  const glowq_status s = latent_check_cache(cache, true);
  if (s != GLOWQ_OK) return s;
  if (T < 1 || T > (1 << 20) || ldc < cache->latent_dim || ldr < cache->rope_dim) return GLOWQ_ERR_SHAPE;
  if (ldc % 8 || ldr % 8) return GLOWQ_ERR_UNSUPPORTED;
  if (!c || !r || !slots) return GLOWQ_ERR_NULL;
  return bad16(c) || bad16(r) || bad4(slots) ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

}  // namespace glowq

using namespace glowq;
extern "C" {

glowq_status glowq_latent_cache_bytes(const glowq_latent_cache* cache, size_t* code_bytes, size_t* scale_bytes, size_t* rope_bytes) {
  if (!code_bytes || !scale_bytes || !rope_bytes) return GLOWQ_ERR_NULL;
  const glowq_status s = latent_check_cache(cache, false);
  if (s != GLOWQ_OK) return s;
  *scale_bytes = (size_t)cache->n_blocks * cache->block_tokens;
  *code_bytes = *scale_bytes * cache->latent_dim;
  *rope_bytes = *scale_bytes * cache->rope_dim * 2;
  return GLOWQ_OK;
}

glowq_status glowq_latent_append(const glowq_latent_cache* cache, const glowq_rope* rope, const glowq_rope_rows* q, const void* c, int32_t ldc,
                                 const void* r, int32_t ldr, const int32_t* slots, const int32_t* positions, int32_t T, void* stream) {
  glowq_status s = check_rows(cache, c, ldc, r, ldr, slots, T);
  if (s != GLOWQ_OK) return s;
  if (!rope && q) return GLOWQ_ERR_NULL;
  if (rope) {
    s = check_rope(rope, cache->rope_dim);
    if (s == GLOWQ_OK && q) s = check_rope_rows(q, 1, cache->rope_dim, cache->act_dtype);
    if (s != GLOWQ_OK) return s;
    if (!positions) return GLOWQ_ERR_NULL;
    if (bad4(positions)) return GLOWQ_ERR_ALIGN;
  }
  return hip_status(launch_latent_append(*cache, rope, q, c, ldc, r, ldr, slots, positions, T, (hipStream_t)stream));
}

glowq_status glowq_latent_gather(const glowq_latent_cache* cache, const int32_t* slots, int32_t T, void* c, int32_t ldc, void* r, int32_t ldr,
                                 void* stream) {
  const glowq_status s = check_rows(cache, c, ldc, r, ldr, slots, T);
  if (s != GLOWQ_OK) return s;
  return hip_status(launch_latent_gather(*cache, slots, T, c, ldc, r, ldr, (hipStream_t)stream));
}

glowq_status glowq_head_maps(const void* x, int32_t ldx, int32_t lhx, const void* w, void* y, int32_t ldy, int32_t lhy, int32_t heads, int32_t d_in,
                             int32_t d_out, int32_t act_dtype, int32_t T, void* stream) {
  if (T < 1 || T > (1 << 20) || heads < 1 || heads > 4096 || d_in < 1 || d_in > 4096 || d_out < 1 || d_out > 4096) return GLOWQ_ERR_SHAPE;
  if (lhx < d_in || lhy < d_out) return GLOWQ_ERR_SHAPE;
  if ((long long)(heads - 1) * lhx + d_in > ldx || (long long)(heads - 1) * lhy + d_out > ldy) return GLOWQ_ERR_SHAPE;
  if (act_dtype != GLOWQ_F16 && act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  if (d_in % 32 || d_out % 16 || ldx % 8 || lhx % 8 || ldy % 8 || lhy % 8) return GLOWQ_ERR_UNSUPPORTED;
  if (!x || !w || !y) return GLOWQ_ERR_NULL;
  if (bad16(x) || bad16(w) || bad16(y)) return GLOWQ_ERR_ALIGN;
  const HeadMapArgs a = {(const uint16_t*)x, (const uint16_t*)w, (uint16_t*)y, ldx, lhx, ldy, lhy, T, d_in, d_out, heads};
  if (act_dtype == GLOWQ_F16) head_maps<ACT_F16>(a, (hipStream_t)stream);
  else head_maps<ACT_BF16>(a, (hipStream_t)stream);
  return hip_status(hipGetLastError());
}

}  // extern "C"
