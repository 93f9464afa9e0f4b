// Attention over the 8-bit cache for many rows per (request, key/value head): prompts and pieces of them.
//
// A workgroup's rows share a tile of 64 keys: its codes are converted once, on their way into LDS, and lie there in operand
// order.  Scores come transposed, S^T = K Q^T, so that a lane holds one row's scores of 16 of 32 keys: maxima and sums stay in
// the lane, and the weights are the second product's operand, O^T = V^T P^T, as they stand.
#pragma once
#include "kv_attend.hpp"

namespace glowq {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
constexpr int MANY_WAVES = 4, MANY_THREADS = 64 * MANY_WAVES, MANY_ROWS = 32 * MANY_WAVES, MANY_STEP = 64;

template <int ACT>
__device__ inline float16_t mfma32(u32x4_t a, u32x4_t b, float16_t c) {
  if constexpr (ACT == ACT_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

template <int DP> struct ManyLds {
  u32x4_t k[2][2][4 * DP][64];       // [buffer][32 keys][16 dims][lane]: key lane & 31, dims 8 (lane >> 5) .. + 8
  u32x4_t v[2][4][2 * DP][64];       // [buffer][16 keys][32 dims][lane]: dim lane & 31, keys 4 h .. + 4 and 8 + 4 h .. + 4, h = lane >> 5
  u32x4_t info[2];                   // [buffer], a word per 16 keys: key scale byte, value scale byte << 8, 1 << 16 if the block is there
  uint32_t odd;                      // a value that is no number came by
  uint32_t arrived;
  KvPart split;
  KvShareLds<MANY_THREADS> share;
};

template <int ACT, int DP>
__device__ inline void kv_many_part(const AttendArgs& a, const KvCrew& crew, const KvPart& pc, const KvRequest& req, ManyLds<DP>& lds) {
  constexpr int NW = MANY_WAVES, R = MANY_ROWS, D = 64 * DP, PER = 8 * DP / NW;      // PER: pieces that a wave brings
  static_assert(NW == 4, "a wave's pieces are of the same 16 keys");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, hf = lane >> 5;
  __builtin_assume(wave >= 0 && wave < NW);
  const KvView& cache = a.cache;
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0);
  const int i0 = row0 / a.group, i1 = (row0 + rows - 1) / a.group;
  const int begin = req.lo(i0, a.window) + max(pc.first, 0) * MANY_STEP;
  const int end = pc.count < 0 ? req.hi(i1) : min(req.hi(i1), begin + pc.count * MANY_STEP);
  const int steps = end > begin ? (end - begin + MANY_STEP - 1) / MANY_STEP : 0;

  // the wave's rows, and their range of positions
  u32x4_t q[4 * DP];
  const int first = row0 + 32 * wave;
  const bool any_row = first < req.rows;
  const int p_row = req.p0 + (first + c32) / a.group;
  const int p_first = req.p0 + first / a.group, p_last = req.p0 + min(first + 31, req.rows - 1) / a.group;
  {
    const int row = first + c32, i = row / a.group;
    const bool live = row < req.rows;
    const uint16_t* src = a.q + (size_t)(req.start + (live ? i : i0)) * a.ldq + ((size_t)pc.head * a.group + (live ? row - i * a.group : 0)) * D + 8 * hf;
#pragma unroll
    for (int s = 0; s < 4 * DP; ++s) q[s] = *(const u32x4_t*)(src + 16 * s);
  }
  float16_t o[2 * DP];
  float m = KV_M_START, l = 0.f;
#pragma unroll
  for (int d = 0; d < 2 * DP; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;

  // What this wave brings: 16 keys, sub, of every tile.  Lane n of `ids` has the block of step n of 64.
  const int sub = wave & 3;
  int ids = 0;
  const auto look_up = [&](int step) {
    const int token = begin + MANY_STEP * (step + lane) + 16 * sub;
    const int id = token < end ? a.table[(size_t)pc.r * a.width + (token >> cache.block_shift)] : -1;
    ids = id >= 0 && id < cache.n_blocks ? id : -1;
  };
  u32x4_t code[PER];
  uint32_t scales = 0;                 // of the tile on its way: key and value scale bytes
  bool there = false;
  const auto fetch = [&](int step) {
    if (step >= steps) return;
    if ((step & 63) == 0) look_up(step);
    int id = __builtin_amdgcn_readlane(ids, step & 63);
    there = id >= 0;
    id = there ? id : 0;
    const int token = begin + MANY_STEP * step + 16 * sub;
    const size_t at = cache.page(id, pc.head) + (there ? (size_t)((token & ((1 << cache.block_shift) - 1)) >> 4) * DP * KV_PIECE : 0);
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int c = wave + NW * n;
      code[n] = *(const u32x4_t*)(cache.codes[c / (4 * DP)] + at + (c / 4 % DP) * KV_PIECE + 16 * lane);
    }
    const size_t sc = (size_t)id * cache.kv_heads + pc.head;
    scales = (uint32_t)cache.scales[0][sc] | (uint32_t)cache.scales[1][sc] << 8;
  };
  const auto stage = [&](int step) {
    if (step >= steps) return;
    const int buf = step & 1, g = lane >> 4, low = lane & 15;
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int c = wave + NW * n, piece = c / 4 % DP;
      if (c < 4 * DP) {
        lds.k[buf][sub >> 1][4 * piece + g][16 * (sub & 1) + low] = kv_operand<ACT>(code[n][0], code[n][1]);
        lds.k[buf][sub >> 1][4 * piece + g][32 + 16 * (sub & 1) + low] = kv_operand<ACT>(code[n][2], code[n][3]);
        continue;
      }
      const uint32_t odd = kv_nan_bytes(code[n][0]) | kv_nan_bytes(code[n][1]) | kv_nan_bytes(code[n][2]) | kv_nan_bytes(code[n][3]);
      if (__any(odd != 0)) {
        // 0 * NaN must not reach rows that do not see it: zeros here, and the rows that do see it get theirs at the end
#pragma unroll
        for (int j = 0; j < 4; ++j) code[n][j] &= ~((kv_nan_bytes(code[n][j]) >> 7) * 0xffu);
        lds.odd = 1;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4_t x = kv_operand<ACT>(code[n][j], code[n][j]);
        ((u32x2_t*)&lds.v[buf][sub][2 * piece + (j >> 1)][32 * (g & 1) + 16 * (j & 1) + low])[g >> 1] = u32x2_t{x[0], x[1]};
      }
    }
    if (wave < 4 && lane == 0) ((uint32_t*)&lds.info[buf])[sub] = scales | (there ? 1u << 16 : 0u);
  };

  if (tid == 0) lds.odd = 0;
  __syncthreads();
  fetch(0);
  stage(0);
  fetch(1);
  __syncthreads();
  for (int step = 0; step < steps; ++step) {
    const int buf = step & 1, t0 = begin + MANY_STEP * step;
    // (waves whose rows see none of these keys, or that have no rows, only bring theirs)
    const bool busy = any_row && t0 <= p_last && (!a.window || t0 + MANY_STEP - 1 > p_first - a.window);
    float16_t s[2];
    if (busy) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
      // operands four at a time, the next four on their way
      u32x4_t x[2][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) x[0][n] = lds.k[buf][0][n][lane];
#pragma unroll
      for (int u = 0; u < 2 * DP; ++u) {
        if (u + 1 < 2 * DP)
#pragma unroll
          for (int n = 0; n < 4; ++n) x[(u + 1) & 1][n] = lds.k[buf][(u + 1) / DP][(u + 1) % DP * 4 + n][lane];
#pragma unroll
        for (int n = 0; n < 4; ++n) s[u / DP] = mfma32<ACT>(x[u & 1][n], q[u % DP * 4 + n], s[u / DP]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    stage(step + 1);
    fetch(step + 2);
    __builtin_amdgcn_sched_barrier(0);
    if (busy) {
      const u32x4_t info = lds.info[buf];
      float ka[4], ve[4], vi[4];
      uint32_t in[4], blocks = 1u << 16;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        in[h] = __builtin_amdgcn_readfirstlane(info[h]);
        ka[h] = kv_pow2((int)(in[h] & 255u) - 127) * a.scale;
        ve[h] = (float)((int)(in[h] >> 8 & 255u) - 127);
        vi[h] = kv_pow2(127 - (int)(in[h] >> 8 & 255u));
        blocks &= in[h];
      }
      if (!(blocks && t0 + MANY_STEP - 1 <= p_first && t0 + MANY_STEP <= end && (!a.window || t0 > p_last - a.window))) {
        const int most = min(end - 1, p_row), least = a.window ? p_row - a.window : -1;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = t0 + 32 * kb + 8 * (e >> 2) + 4 * hf + (e & 3);
            s[kb][e] = key <= most && key > least && (in[2 * kb + (e >> 3)] & 1u << 16) ? s[kb][e] : -INFINITY;
          }
      }
      float most = -INFINITY;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        float t = s[h >> 1][8 * (h & 1)];
#pragma unroll
        for (int e = 1; e < 8; ++e) t = fmaxf(t, s[h >> 1][8 * (h & 1) + e]);
        most = fmaxf(most, __builtin_fmaf(t, ka[h], ve[h]));
      }
      if (__any(most > m + KV_M_SLACK)) {
        most = fmaxf(fmaxf(most, __shfl_xor(most, 32, 64)), m);
        const float f = __builtin_amdgcn_exp2f(m - most);
        m = most;
        l *= f;
#pragma unroll
        for (int d = 0; d < 2 * DP; ++d) o[d] *= f;
      }
      u32x4_t p[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const float c = ve[h] - m;
        float e[8], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h >> 1][8 * (h & 1) + i], ka[h], c));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[h][i] = kv_pack<ACT>(e[2 * i], e[2 * i + 1]);
          sum = kv_add2<ACT>(p[h][i], sum);
        }
        l = __builtin_fmaf(sum, vi[h], l);
      }
      __builtin_amdgcn_sched_barrier(0);
      u32x4_t y[2][2 * DP];
#pragma unroll
      for (int d = 0; d < 2 * DP; ++d) y[0][d] = lds.v[buf][0][d][lane];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        if (h + 1 < 4)
#pragma unroll
          for (int d = 0; d < 2 * DP; ++d) y[(h + 1) & 1][d] = lds.v[buf][h + 1][d][lane];
#pragma unroll
        for (int d = 0; d < 2 * DP; ++d) o[d] = mfma32<ACT>(y[h & 1][d], p[h], o[d]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();
  }
  if (lds.odd) {
    // values that are no numbers: every dim of every key of the piece is looked at again, for the rows that see the key
    for (int key = begin; key < end; ++key) {
      const int id = a.table[(size_t)pc.r * a.width + (key >> cache.block_shift)];
      if (id < 0 || id >= cache.n_blocks) continue;
      const uint8_t* const page = cache.codes[1] + cache.page(id, pc.head);
#pragma unroll
      for (int d = 0; d < 2 * DP; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((page[kv_value_byte(key & ((1 << cache.block_shift) - 1), 32 * d + 8 * (e >> 2) + 4 * hf + (e & 3), cache.dim_shift)] & 0x7f) == 0x7f)
            if (key <= p_row && (!a.window || key > p_row - a.window)) o[d][e] = NAN;
    }
  }

  const bool split = pc.parts > 1;
  float* const slot = split ? crew.slots + (size_t)pc.slot * (R * (D + 2)) : nullptr;
  const int at = 32 * wave + c32, row = row0 + at;
  const float sum = l + __shfl_xor(l, 32, 64);
  const float inv = !split ? kv_inverse(sum, a, req, row) : sum != 0.f ? 1.f / sum : 0.f;
  const bool live = at < rows;
  const int i = row / a.group;
  uint16_t* const to = a.out + (size_t)(req.start + i) * a.ldo + ((size_t)pc.head * a.group + (row - i * a.group)) * D;
#pragma unroll
  for (int d = 0; d < 2 * DP; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 8) {
      const float4_t x = float4_t{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]} * inv;
      const float4_t y = float4_t{o[d][e + 4], o[d][e + 5], o[d][e + 6], o[d][e + 7]} * inv;
      if (!split) {
        // lanes 32 apart exchange halves: eight dims in a row each
        const auto lo = __builtin_amdgcn_permlane32_swap(kv_pack<ACT>(x[0], x[1]), kv_pack<ACT>(y[0], y[1]), false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(kv_pack<ACT>(x[2], x[3]), kv_pack<ACT>(y[2], y[3]), false, false);
        if (live) *(u32x4_t*)(to + 32 * d + 2 * e + 8 * hf) = u32x4_t{lo[0], hi[0], lo[1], hi[1]};
      } else if (live) {
        store16_device(slot + at * D + 32 * d + 2 * e + 4 * hf, __builtin_bit_cast(u32x4_t, x));
        store16_device(slot + at * D + 32 * d + 2 * e + 8 + 4 * hf, __builtin_bit_cast(u32x4_t, y));
      }
    }
  if (!split) return;
  if (live && hf == 0) {
    kv_store_device(slot + R * D + at, m);
    kv_store_device(slot + R * (D + 1) + at, sum);
  }
  if (tid == 0) lds.split = pc;
  kv_arrive<MANY_THREADS>(crew, &lds.split, 1, &lds.arrived);
  if (lds.arrived == (uint32_t)pc.parts - 1) kv_join<ACT, D, R, MANY_THREADS>(a, crew, req, pc, row0, rows, (float*)&lds);
}

template <int ACT, int DP>
__device__ inline void kv_many(const AttendArgs& a, const KvCrew& crew, int wg, ManyLds<DP>& lds) {
  KvShare share = kv_share<MANY_THREADS, MANY_ROWS, MANY_STEP>(a, crew, wg, lds.share);
  for (;;) {
    KvRequest req;
    const KvPart pc = kv_next<MANY_THREADS, MANY_ROWS, MANY_STEP>(a, crew, share, req, lds.share);
    if (pc.r < 0) return;
    kv_many_part<ACT, DP>(a, crew, pc, req, lds);
    __syncthreads();                       // the words that a part leaves in LDS have been read
  }
}

}  // namespace glowq
