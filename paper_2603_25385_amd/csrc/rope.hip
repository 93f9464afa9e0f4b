// Rotary positions: frequencies, rows rotated in memory, keys rotated on their way into the 8-bit cache.
#include <algorithm>
#include <cmath>
#include "kv_append.hpp"
#include "kv_host.hpp"
#include "rope_host.hpp"

namespace glowq {

// ---------------------------------------------------------------------------------------
// Rows.  Bytes in and out are the bound; for single tokens the launch and the chain position, angle, store.
constexpr int ROTATE_THREADS = 256, ROTATE_PER = 8;
constexpr long long MOST_THREADS = 0xffffffffll - ROTATE_THREADS;       // a launch counts its threads in 32 bits

template <int TYPE> __global__ void __launch_bounds__(ROTATE_THREADS) k_rotate(RotateArgs a) {
  rope_rotate<TYPE>(a, (long long)blockIdx.x * ROTATE_THREADS + threadIdx.x);
}

RotateArgs make_rotate_args(const glowq_rope& rope, const glowq_rope_rows* rows, int n_rows, int dim, int dtype, const int32_t* positions, int T,
                            long long* threads) {
  const long long size = dtype == GLOWQ_F32 ? 4 : 2;       // (strides in bytes outgrow 32 bits)
  RotateArgs a = {};
  a.rope = rope_view(rope);
  for (int n = 0; n < ROPE_TENSORS; ++n) {
    if (n < n_rows) {
      const glowq_rope_rows& r = rows[n];
      a.heads += r.heads;
      a.t[n] = RopeTensor{(const char*)r.x, (char*)r.y, r.ldx * size, r.ldy * size, r.lhx * size, r.lhy * size, a.heads};
    } else a.t[n].end = 0x7fffffff;
  }
  a.positions = positions;
  a.T = T;
  a.units = (int)(dim * size / 32);
  // heads of a thread: as many as leave the machine full of threads, up to eight, so that angles are made once for them
  const long long all = (long long)T * a.heads * a.units;
  a.per = (int)std::min<long long>(ROTATE_PER, std::max<long long>(1, all >> 18));
  a.groups = (a.heads + a.per - 1) / a.per;
  *threads = (long long)T * a.groups * a.units;
  return a;
}

// Threads of a large call (all >> 18 above the heads of a thread: others have fewer than 2^22)
long long rope_threads(const glowq_rope_rows* rows, int n_rows, int dim, int dtype, int T) {
  long long heads = 0;
  for (int n = 0; n < n_rows; ++n) heads += rows[n].heads;
  return (long long)T * ((heads + ROTATE_PER - 1) / ROTATE_PER) * (dim * (dtype == GLOWQ_F32 ? 4 : 2) / 32);
}

static hipError_t launch_rotate(const glowq_rope& rope, const glowq_rope_rows* rows, int n_rows, int dim, int dtype, const int32_t* positions, int T,
                                hipStream_t st) {
  long long threads;
  const RotateArgs a = make_rotate_args(rope, rows, n_rows, dim, dtype, positions, T, &threads);
  const dim3 grid((unsigned)((threads + ROTATE_THREADS - 1) / ROTATE_THREADS)), block(ROTATE_THREADS);
  if (dtype == GLOWQ_F16) k_rotate<GLOWQ_F16><<<grid, block, 0, st>>>(a);
  else if (dtype == GLOWQ_BF16) k_rotate<GLOWQ_BF16><<<grid, block, 0, st>>>(a);
  else k_rotate<GLOWQ_F32><<<grid, block, 0, st>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// Keys rotated on their way into the cache, values beside them, and q.  The rotated keys are never rounded to 16 bits: block
// exponent and codes come from their fp32 values.  A launch has workgroups for keys (a wave per run of tokens and head; the
// angles of a run are made once, in LDS, by all four waves, for all heads that they take), for values (as glowq_kv_append) and for q.
struct AppendRotatedArgs {
  KvView cache;
  const uint16_t* rows[2];
  long long ld[2];
  const int32_t *slots, *positions;
  RotateArgs q;
  RopeView rope;
  int T, per;
  int key_groups, heads_per_wave;      // workgroups that share out the heads' keys, heads that a wave takes one after another
  int value_groups;
  int q_blocks;                        // workgroups for q behind those
  int row_blocks;
};

// Four numbers over 2^e as codes
__device__ inline uint32_t kv_encode4_scaled(float a, float b, float c, float d, float grid) {
  typedef short short2_t __attribute__((ext_vector_type(2)));
  short2_t w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, grid, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, grid, true);
  return __builtin_bit_cast(uint32_t, w);
}

// TOKENS: of a run at once (32 where blocks are no larger: half the registers and LDS; four prompts of up to 2100 tokens, 32 heads,
// read-back included: 136 -> 128 us, 117 with four waves a SIMD)
template <int ACT, int DP, int TOKENS>
__device__ inline void append_rotated_keys(const AppendRotatedArgs& a, int group, float4_t (*table)[4][4 * DP]) {
  constexpr int D = 64 * DP, UNITS = D / 16, TILE = 16 * D, PER = 64 / UNITS, LOADS = TOKENS / PER;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const KvView& c = a.cache;
  const int B = 1 << c.block_shift, unit = lane % UNITS, token = lane / UNITS;
  const bool turn = unit < a.rope.units;
  const int da = a.rope.dim_a(unit), db = a.rope.dim_b(unit);
  // (all four waves see the same runs, so that barriers inside are met by all)
  kv_runs(c, a.slots, a.T, a.per, [&](int first, int slot, int m) {
    const int block = slot >> c.block_shift, off = slot & (B - 1), end = off + m;
    const auto stretch = [&](int from) { return min(end, (from & ~15) + TOKENS); };
    const bool once = stretch(off) == end;
    // the angles of tokens from .. to of the block: [token][c0-3, c4-7, s0-3, s4-7][unit]
    const auto angles = [&](int from, int to) {
      __syncthreads();                     // (nobody reads those before)
      const int pairs = 8 * a.rope.units;
      for (int i = tid; i < (to - from) * pairs; i += RUN_THREADS) {
        const int t = i / pairs, pair = i - t * pairs;
        float cs, sn;
        rope_angle(a.rope.turns[pair], max(a.positions[first + from - off + t], 0), a.rope.magnitude, cs, sn);
        ((float*)&table[t][(pair & 7) >> 2][pair >> 3])[pair & 3] = cs;
        ((float*)&table[t][2 + ((pair & 7) >> 2)][pair >> 3])[pair & 3] = sn;
      }
      __syncthreads();
    };
    if (once) angles(off, end);
    for (int k = 0; k < a.heads_per_wave; ++k) {
      const int head = (group * a.heads_per_wave + k) * RUN_WAVES + wave;
      const bool live = head < c.kv_heads;
      const int h = live ? head : 0;
      const uint16_t* const src = a.rows[0] + (size_t)h * D;
      uint8_t* const scale = c.scales[0] + (size_t)block * c.kv_heads + h;
      uint8_t* const page = c.codes[0] + c.page(block, h);
      const int byte = *scale;
      u32x4_t x[LOADS][2];
      const auto load = [&](int from, int to) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int t = from + token + i * PER;
          x[i][0] = x[i][1] = u32x4_t{0, 0, 0, 0};
          if (t < to) {
            const uint16_t* p = src + (size_t)(first + t - off) * a.ld[0];
            x[i][0] = *(const u32x4_t*)(p + da);
            x[i][1] = *(const u32x4_t*)(p + db);
          }
        }
      };
      // token from + token + i PER, rotated
      const auto rotated = [&](int i, float (&u)[8], float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = kv_act_f32<ACT>(x[i][0][e >> 1] >> (16 * (e & 1)) & 0xffffu);
          v[e] = kv_act_f32<ACT>(x[i][1][e >> 1] >> (16 * (e & 1)) & 0xffffu);
        }
        if (turn) {
          const auto& at = table[token + i * PER];
          float cs[8], sn[8];
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              cs[4 * q + e] = at[q][unit][e];
              sn[4 * q + e] = at[2 + q][unit][e];
            }
          rope_turn_unit(u, v, cs, sn, a.rope.pairs);
        }
      };
      uint32_t top = 0;
      for (int from = off; from < end; from = stretch(from)) {
        const int to = stretch(from);
        if (!once) angles(from, to);
        load(from, to);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          if (from + i * PER >= to) continue;
          float u[8], v[8];
          rotated(i, u, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t mu = __builtin_bit_cast(uint32_t, u[e]) & 0x7fffffffu, mv = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
            if (from + token + i * PER < to) {       // (what is no number does not count)
              top = mu < 0x7f800000u ? max(top, mu) : top;
              top = mv < 0x7f800000u ? max(top, mv) : top;
            }
          }
        }
      }
      for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
      const int before = off > 0 ? min(byte - 127, 126) : KV_EXP_MIN;
      const int e = max(before, kv_exponent(top));
      const float grid = kv_pow2(e), shrink = kv_pow2(max(before - e, -126));
      const bool grown = off > 0 && e > before;
      if (live && lane == 0 && (off == 0 || grown)) *scale = (uint8_t)(e + 127);
      if (live && grown)                   // older tokens of the block to the new grid
        for (int u = lane; u < ((off + 15) >> 4) * (TILE / 16); u += 64) {
          if (u / (TILE / 16) * 16 + (u & 15) >= off) continue;
          u32x4_t w = ((u32x4_t*)page)[u];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = kv_recode4(w[i], shrink);
          ((u32x4_t*)page)[u] = w;
        }
      for (int from = off; from < end; from = stretch(from)) {
        const int to = stretch(from);
        if (!once) {
          angles(from, to);
          load(from, to);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int t = from + token + i * PER;
          if (!live || t >= to) continue;
          float u[8], v[8];
          rotated(i, u, v);
          typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
          *(u32x2_t*)(page + kv_key_byte(t, da, 6 + (DP == 2))) = u32x2_t{kv_encode4_scaled(u[0], u[1], u[2], u[3], grid), kv_encode4_scaled(u[4], u[5], u[6], u[7], grid)};
          *(u32x2_t*)(page + kv_key_byte(t, db, 6 + (DP == 2))) = u32x2_t{kv_encode4_scaled(v[0], v[1], v[2], v[3], grid), kv_encode4_scaled(v[4], v[5], v[6], v[7], grid)};
        }
      }
    }
  }, [](int) {});
}

template <int ACT, int DP, int TOKENS>
__global__ void __launch_bounds__(RUN_THREADS, DP == 2 && TOKENS == 64 ? 3 : 4) k_kv_append_rotated(AppendRotatedArgs a) {
  __shared__ union {
    float4_t table[TOKENS][4][4 * DP];
    u32x4_t image[RUN_WAVES][TOKENS * DP * 4];
  } lds;
  const int group = blockIdx.y;
  if (group < a.key_groups) {
    append_rotated_keys<ACT, DP, TOKENS>(a, group, lds.table);
  } else if (group < a.key_groups + a.value_groups) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = (group - a.key_groups) * RUN_WAVES + wave;
    if (head >= a.cache.kv_heads) return;
    const uint16_t* const src = a.rows[1] + (size_t)head * 64 * DP;
    kv_runs(a.cache, a.slots, a.T, a.per, [&](int first, int slot, int m) {
      kv_append_run<ACT, DP, TOKENS>(a.cache, 1, head, src, a.ld[1], lds.image[wave], first, slot, m);
    }, [](int) {});
  } else {
    const long long block = (long long)(group - a.key_groups - a.value_groups) * a.row_blocks + blockIdx.x;
    if (block < a.q_blocks) rope_rotate<ACT>(a.q, block * RUN_THREADS + threadIdx.x);
  }
}

static hipError_t launch_append_rotated(const glowq_kv_cache& cache, const glowq_rope& rope, const glowq_rope_rows* q, const void* k, int ldk, const void* v,
                                        int ldv, int act, const int32_t* slots, const int32_t* positions, int T, hipStream_t st) {
  AppendRotatedArgs a = {};
  a.cache = kv_view(cache);
  a.rows[0] = (const uint16_t*)k;
  a.rows[1] = (const uint16_t*)v;
  a.ld[0] = ldk;
  a.ld[1] = ldv;
  a.slots = slots;
  a.positions = positions;
  a.rope = rope_view(rope);
  a.T = T;
  a.per = rows_per_wave(T, cache.kv_heads);
  a.row_blocks = (T + a.per - 1) / a.per;
  // heads of a wave: two share the angles where runs are many
  a.heads_per_wave = a.per > 1 && cache.kv_heads > RUN_WAVES ? 2 : 1;
  a.key_groups = (cache.kv_heads + RUN_WAVES * a.heads_per_wave - 1) / (RUN_WAVES * a.heads_per_wave);
  a.value_groups = (cache.kv_heads + RUN_WAVES - 1) / RUN_WAVES;
  int q_groups = 0;
  if (q) {
    long long threads;
    a.q = make_rotate_args(rope, q, 1, cache.head_dim, act, positions, T, &threads);
    a.q_blocks = (int)((threads + RUN_THREADS - 1) / RUN_THREADS);
    q_groups = (a.q_blocks + a.row_blocks - 1) / a.row_blocks;
  }
  const dim3 grid(a.row_blocks, a.key_groups + a.value_groups + q_groups), block(RUN_THREADS);
#define GLOWQ_APPEND(DP, TOKENS) \
  act == GLOWQ_F16 ? k_kv_append_rotated<ACT_F16, DP, TOKENS><<<grid, block, 0, st>>>(a) : k_kv_append_rotated<ACT_BF16, DP, TOKENS><<<grid, block, 0, st>>>(a)
  if (cache.head_dim == 64) cache.block_tokens <= 32 ? (GLOWQ_APPEND(1, 32)) : (GLOWQ_APPEND(1, 64));
  else cache.block_tokens <= 32 ? (GLOWQ_APPEND(2, 32)) : (GLOWQ_APPEND(2, 64));
#undef GLOWQ_APPEND
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------
// Argument checks
static bool bad16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
static bool bad4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

glowq_status check_rope(const glowq_rope* rope, int head_dim) {
  if (!rope) return GLOWQ_ERR_NULL;
  if (rope->rotary_dim < 2 || rope->rotary_dim % 2 || rope->rotary_dim > head_dim) return GLOWQ_ERR_SHAPE;
  if (rope->layout != GLOWQ_ROPE_HALVES && rope->layout != GLOWQ_ROPE_PAIRS) return GLOWQ_ERR_SHAPE;
  if (!(std::fabs(rope->magnitude) <= 3e38f)) return GLOWQ_ERR_SHAPE;
  if (rope->rotary_dim % 16) return GLOWQ_ERR_UNSUPPORTED;
  if (!rope->turns) return GLOWQ_ERR_NULL;
  return (uintptr_t)rope->turns & 7u ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

glowq_status check_rope_rows(const glowq_rope_rows* rows, int n_rows, int dim, int dtype) {
  if (!rows) return GLOWQ_ERR_NULL;
  if (n_rows < 1 || n_rows > ROPE_TENSORS) return GLOWQ_ERR_SHAPE;
  for (int n = 0; n < n_rows; ++n) {
    const glowq_rope_rows& r = rows[n];
    if (r.heads < 1 || r.heads > 4096 || r.lhx < dim || r.lhy < dim) return GLOWQ_ERR_SHAPE;
    if ((long long)(r.heads - 1) * r.lhx + dim > r.ldx || (long long)(r.heads - 1) * r.lhy + dim > r.ldy) return GLOWQ_ERR_SHAPE;
    if (r.ldx % 8 || r.lhx % 8 || r.ldy % 8 || r.lhy % 8) return GLOWQ_ERR_UNSUPPORTED;
    if (!r.x || !r.y) return GLOWQ_ERR_NULL;
    if (bad16(r.x) || bad16(r.y)) return GLOWQ_ERR_ALIGN;
    // in place, every number stays where it is
    if (r.x == r.y && (r.ldx != r.ldy || r.lhx != r.lhy)) return GLOWQ_ERR_SHAPE;
  }
  return GLOWQ_OK;
}

}  // namespace glowq

using namespace glowq;
extern "C" {

glowq_status glowq_rope_turns(const glowq_rope_spec* spec, uint64_t* turns, float* magnitude) {
  if (!spec || !turns || !magnitude) return GLOWQ_ERR_NULL;
  const int r = spec->rotary_dim;
  if (r < 2 || r % 2 || r > 4096 || !(spec->base > 1.0) || !std::isfinite(spec->base)) return GLOWQ_ERR_SHAPE;
  if (spec->scaling < GLOWQ_ROPE_PLAIN || spec->scaling > GLOWQ_ROPE_RAMP) return GLOWQ_ERR_SHAPE;
  const bool banded = spec->scaling == GLOWQ_ROPE_BANDS || spec->scaling == GLOWQ_ROPE_RAMP;
  if (spec->scaling != GLOWQ_ROPE_PLAIN && (!(spec->factor >= 1.0) || !std::isfinite(spec->factor))) return GLOWQ_ERR_SHAPE;
  if (banded && (!(spec->low > 0.0) || !(spec->high > spec->low) || !std::isfinite(spec->high) || spec->trained_length < 1)) return GLOWQ_ERR_SHAPE;
  if (spec->scaling == GLOWQ_ROPE_REBASED && r == 2) return GLOWQ_ERR_SHAPE;             // (its exponent r / (r - 2))
  if (r % 16) return GLOWQ_ERR_UNSUPPORTED;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  const long double factor = spec->factor, length = spec->trained_length;
  long double base = spec->base;
  if (spec->scaling == GLOWQ_ROPE_REBASED) base *= powl(factor, (long double)r / (r - 2));
  long double first = 0, last = 0;
  if (spec->scaling == GLOWQ_ROPE_RAMP) {
    // the (real) index of the pair that makes so many turns over the trained length
    const auto where = [&](long double turns_made) { return r * logl(length / (turns_made * two_pi)) / (2 * logl(base)); };
    first = std::max(floorl(where(spec->high)), 0.0L);
    last = std::min(ceill(where(spec->low)), (long double)(r - 1));
  }
  for (int i = 0; i < r / 2; ++i) {
    long double f = powl(base, -2.0L * i / r);
    if (spec->scaling == GLOWQ_ROPE_STRETCHED) f /= factor;
    if (banded) {
      long double slow;                    // the share of f / factor
      if (spec->scaling == GLOWQ_ROPE_RAMP) slow = (i - first) / std::max(last - first, 0.001L);
      else slow = 1 - (length * f / two_pi - spec->low) / ((long double)spec->high - spec->low);
      slow = std::min(std::max(slow, 0.0L), 1.0L);
      f = slow * f / factor + (1 - slow) * f;
    }
    turns[i] = (uint64_t)(f / two_pi * 18446744073709551616.0L + 0.5L);       // (f <= 1: far below 2^64)
  }
  *magnitude = spec->scaling == GLOWQ_ROPE_RAMP ? (float)(0.1L * logl(factor) + 1) : 1.f;
  return GLOWQ_OK;
}

glowq_status glowq_rotate(const glowq_rope* rope, const glowq_rope_rows* rows, int32_t n_rows, int32_t head_dim, int32_t dtype,
                          const int32_t* positions, int32_t T, void* stream) {
  if (head_dim < 1 || head_dim > 4096 || T < 1 || T > (1 << 20)) return GLOWQ_ERR_SHAPE;
  glowq_status s = check_rope(rope, head_dim);
  if (s != GLOWQ_OK) return s;
  if (dtype != GLOWQ_F16 && dtype != GLOWQ_BF16 && dtype != GLOWQ_F32) return GLOWQ_ERR_DTYPE;
  if (head_dim % 16) return GLOWQ_ERR_UNSUPPORTED;
  s = check_rope_rows(rows, n_rows, head_dim, dtype);
  if (s != GLOWQ_OK) return s;
  if (!positions) return GLOWQ_ERR_NULL;
  if (bad4(positions)) return GLOWQ_ERR_ALIGN;
  if (rope_threads(rows, n_rows, head_dim, dtype, T) > MOST_THREADS) return GLOWQ_ERR_SHAPE;
  return hip_status(launch_rotate(*rope, rows, n_rows, head_dim, dtype, positions, T, (hipStream_t)stream));
}

glowq_status glowq_kv_append_rotated(const glowq_kv_cache* cache, const glowq_rope* rope, const glowq_rope_rows* q, const void* k, int32_t ldk,
                                     const void* v, int32_t ldv, int32_t act_dtype, const int32_t* slots, const int32_t* positions, int32_t T,
                                     void* stream) {
  glowq_status s = kv_check_rows(cache, k, ldk, v, ldv, slots, T);
  if (s != GLOWQ_OK) return s;
  if (act_dtype != GLOWQ_F16 && act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  s = check_rope(rope, cache->head_dim);
  if (s == GLOWQ_OK && q) s = check_rope_rows(q, 1, cache->head_dim, act_dtype);
  if (s != GLOWQ_OK) return s;
  if (!positions) return GLOWQ_ERR_NULL;
  if (bad4(positions)) return GLOWQ_ERR_ALIGN;
  return hip_status(launch_append_rotated(*cache, *rope, q, k, ldk, v, ldv, act_dtype, slots, positions, T, (hipStream_t)stream));
}

}  // extern "C"
