// Attention over the 8-bit cache for many rows per (request, key/value head): prompts and pieces of them.
//
// A workgroup's 128 rows share tiles of 64 keys, which direct loads bring into LDS as they lie in the cache, three tiles ahead;
// every wave converts what it reads.  (Converted once on their way into LDS the codes took twice the bytes there and a chain of
// waits: an 8000-token prompt 570 us, 555 so.)  An 8000-token prompt of 32 heads takes 550 to 570 us, 0.93 PFLOP/s: matrix pipe busy
// 0.41, vector ALU 0.64, which a product keeps from issuing for half its time.  Scores come transposed, S^T = K Q^T (32x32x16),
// so that a lane holds 16 of 32 keys of one row: sums stay in the lane, and the weights are the second product's operand, O^T = V^T P^T, as they stand.  The
// contractions' order is the cache's: a lane's 16 bytes of keys are 16 dims in a row, operands of two instructions; its 16
// bytes of values are four dims 16 apart of four keys, operands of four instructions, each of which has 32 dims
// d + 16 j + 64 x of its lanes (d, x).
#pragma once
#include "kv_attend.hpp"

namespace glowq {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
constexpr int MANY_WAVES = 4, MANY_THREADS = 64 * MANY_WAVES, MANY_ROWS = 32 * MANY_WAVES, MANY_STEP = 64;
constexpr int MANY_STAGES = 4;

template <int ACT>
__device__ inline float16_t mfma32(u32x4_t a, u32x4_t b, float16_t c) {
  if constexpr (ACT == ACT_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

template <int DP> struct ManyLds {
  uint8_t k[MANY_STAGES][4][DP][KV_PIECE];        // [stage][16 keys][64 dims]
  uint8_t v[MANY_STAGES][4][DP][KV_PIECE];
  uint32_t odd, found;               // a result that is no number: the part is done again; a value that is none
  uint32_t arrived;
};

template <int ACT, int DP>
__device__ inline void kv_many_part(const AttendArgs& a, const KvCrew& crew, const KvPart& pc, const KvRequest& req, ManyLds<DP>& lds) {
  constexpr int R = MANY_ROWS, D = 64 * DP, PER = 2 * DP;         // PER: pieces that a wave brings of a tile
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, hf = lane >> 5;
  const KvView& cache = a.cache;
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0);
  const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int i0 = scalar(row0 / a.group), i1 = scalar((row0 + rows - 1) / a.group);
  const int begin = req.lo(i0, a.window) + pc.first * MANY_STEP;
  const int end = min(req.hi(i1), begin + pc.count * MANY_STEP);
  const int steps = end > begin ? (end - begin + MANY_STEP - 1) / MANY_STEP : 0;

  // the wave's rows, and their range of positions
  u32x4_t q[4 * DP];                 // dims 32 u + 16 hf .. + 8 and the next 8
  const int first = row0 + 32 * wave;
  const bool any_row = first < req.rows;
  const int p_row = req.p0 + (first + c32) / a.group;
  const int p_first = req.p0 + scalar(first / a.group), p_last = req.p0 + scalar(min(first + 31, req.rows - 1) / a.group);
  {
    const int row = first + c32, i = row / a.group;
    const bool live = row < req.rows;
    const uint16_t* src = a.q + (size_t)(req.start + (live ? i : i0)) * a.ldq + ((size_t)pc.head * a.group + (live ? row - i * a.group : 0)) * D + 16 * hf;
#pragma unroll
    for (int u = 0; u < 2 * DP; ++u) {
      q[2 * u] = *(const u32x4_t*)(src + 32 * u);
      q[2 * u + 1] = *(const u32x4_t*)(src + 32 * u + 8);
    }
  }
  float16_t o[2 * DP];
  float m, l;
  KvReference ref;

  // Lane 4 n + s: block of 16 keys s of step 16 w + n, and its scales, for the window w at hand and the one behind it.  The
  // next window's are looked up half a window ahead, in three moves.  Keys that no row sees count as not there: nobody need have
  // written their block.
  struct Scales {
    float key, value;                  // key scale times the scores', 2^(exponent - E)
    int exponent, bytes[2];            // of the values; as the cache has them
    unsigned long long wild;           // lanes whose values need more than that
  };
  int ids, ids_next;
  Scales at_hand, behind;
  const auto place = [&](Scales& x) {
    x.value = kv_value_scale(x.exponent, ref.at);
    x.wild = __ballot(kv_wild<ACT>(x.exponent, ref.at));
  };
  const auto look_up = [&](int window) {
    const int token = begin + MANY_STEP * (16 * window + (lane >> 2)) + 16 * (lane & 3);
    const bool seen = token < end && (!a.window || token + 15 > req.p0 + i0 - a.window);
    const int id = seen ? a.table[(size_t)pc.r * a.width + (token >> cache.block_shift)] : -1;
    return id < cache.n_blocks ? id : -1;
  };
  const auto look_up_scales = [&](int id, Scales& x) {
    const size_t sc = (size_t)max(id, 0) * cache.kv_heads + pc.head;
    x.exponent = id < 0 ? KV_ABSENT : 0;
    x.bytes[0] = cache.scales[0][sc];
    x.bytes[1] = cache.scales[1][sc];
  };
  // (apart, since it waits for the bytes: nothing is made of those that were read for a block that is not there)
  const auto settle = [&](Scales& x) {
    const int e = x.bytes[1] - 127;
    x.key = x.exponent == KV_ABSENT ? 1.f : kv_pow2(x.bytes[0] - 127) * a.scale;
    x.exponent = x.exponent == KV_ABSENT ? KV_ABSENT : e < KvRange<ACT>::ZERO ? KV_ZEROS : e;
    place(x);
  };
  // the wave's pieces of a tile, 16 keys, into LDS
  const auto bring = [&](int step) {
    const int n = 4 * (step & 15) + wave, stage = step % MANY_STAGES, token = begin + MANY_STEP * step + 16 * wave;
    const int id = ((step >> 4) & 1) == 0 ? __builtin_amdgcn_readlane(ids, n) : __builtin_amdgcn_readlane(ids_next, n);
    const bool there = id >= 0;
    const size_t at = cache.page(there ? id : 0, pc.head) + (there ? (size_t)((token & ((1 << cache.block_shift) - 1)) >> 4) * DP * KV_PIECE : 0) + 16 * lane;
#pragma unroll
    for (int d = 0; d < DP; ++d) {
      lds_dma16(cache.codes[0] + at + d * KV_PIECE, lds_address(&lds.k[stage][wave][d][0]));
      lds_dma16(cache.codes[1] + at + d * KV_PIECE, lds_address(&lds.v[stage][wave][d][0]));
    }
  };

  // One tile.  Values behind the last key or in blocks that are not there, and in a second pass values that are no numbers, are
  // taken as zeros.
  bool again = false;
  const auto tile = [&](int step, float (&ka)[4], float (&vs)[4], uint32_t wild, const auto exponent) __attribute__((always_inline)) {
    const int t0 = begin + MANY_STEP * step, stage = step % MANY_STAGES;
    uint32_t gone = 0;                     // of the keys, which 16 are not there
    if (__builtin_expect(wild != 0, 0))
#pragma unroll
      for (int h = 0; h < 4; ++h) gone |= (exponent(h) == KV_ABSENT ? 1u : 0u) << h;
    const bool clean = again || gone || t0 + MANY_STEP > end;
    // keys: 16 bytes of a lane, two instructions.  Two sums in turn: one waits twice as long for itself as an instruction takes
    const uint8_t* const kp = &lds.k[stage][c32 >> 4][0][(16 * hf + (c32 & 15)) * 16];
    float16_t s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
    u32x4_t x[2][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) x[0][kb] = *(const u32x4_t*)(kp + 2 * kb * DP * KV_PIECE);
#pragma unroll
    for (int u = 0; u < 2 * DP; ++u) {
      if (u + 1 < 2 * DP)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) x[(u + 1) & 1][kb] = *(const u32x4_t*)(kp + (2 * kb * DP + ((u + 1) >> 1)) * KV_PIECE + ((u + 1) & 1) * 512);
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          s[kb] = mfma32<ACT>(kv_operand<ACT>(x[u & 1][kb][2 * half], x[u & 1][kb][2 * half + 1]), q[2 * u + half], s[kb]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (gone || !(t0 + MANY_STEP - 1 <= p_first && t0 + MANY_STEP <= end && (!a.window || t0 > p_last - a.window))) {
      const int most = min(end - 1, p_row), least = a.window ? p_row - a.window : -1;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = t0 + 32 * kb + 8 * (e >> 2) + 4 * hf + (e & 3);
          s[kb][e] = key <= most && key > least && !(gone >> (2 * kb + (e >> 3)) & 1) ? s[kb][e] * ka[2 * kb + (e >> 3)] : -INFINITY;
        }
#pragma unroll
      for (int h = 0; h < 4; ++h) ka[h] = 1.f;   // (in the scores already: a scale may be 0 in fp32, and -inf times 0 is no number)
    }
    float most = -INFINITY;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      float t = s[h >> 1][8 * (h & 1)];
#pragma unroll
      for (int e = 1; e < 8; ++e) t = fmaxf(t, s[h >> 1][8 * (h & 1) + e]);
      most = fmaxf(most, t * ka[h]);
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
      float e[8], sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h >> 1][8 * (h & 1) + i], ka[h], -m));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[h][i] = kv_pack<ACT>(e[2 * i], e[2 * i + 1]);
        sum = kv_add2<ACT>(p[h][i], sum);
      }
      l += sum;
    }
    __builtin_amdgcn_sched_barrier(0);
    // values: keys 4 hf .. + 4 and 8 + 4 hf .. + 4 of each 16
    const int before = ref.at;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      if (__builtin_expect(wild >> h & 1, 0)) {
        const int e = exponent(h);
        if (e > KV_ZEROS && kv_wild<ACT>(e, ref.at)) {
          kv_refer(e, ref, [&](int by) {
#pragma unroll
            for (int d = 0; d < 2 * DP; ++d)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[d][i] = __builtin_ldexpf(o[d][i], by);
          });
          wild = 15;                       // (scales of the rest were made for the old one)
        }
        vs[h] = kv_value_scale(e, ref.at);
      }
      const uint8_t* const vp = &lds.v[stage][h][DP == 2 ? c32 >> 4 : 0][(16 * hf + (c32 & 15)) * 16 + (DP == 2 ? 0 : 8 * (c32 >> 4))];
      uint32_t w[2][2 * DP];
      if constexpr (DP == 2) {
        const u32x4_t lo = *(const u32x4_t*)vp, hi = *(const u32x4_t*)(vp + 512);
#pragma unroll
        for (int j = 0; j < 4; ++j) { w[0][j] = lo[j]; w[1][j] = hi[j]; }
      } else {
        const u32x2_t lo = *(const u32x2_t*)vp, hi = *(const u32x2_t*)(vp + 512);
#pragma unroll
        for (int j = 0; j < 2; ++j) { w[0][j] = lo[j]; w[1][j] = hi[j]; }
      }
      if (clean)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int left = gone >> h & 1 ? 0 : min(4, end - (t0 + 16 * h + 8 * y + 4 * hf));
          const uint32_t keep = left > 0 ? 0xffffffffu >> (8 * (4 - left)) : 0u;
#pragma unroll
          for (int j = 0; j < 2 * DP; ++j) {
            w[y][j] &= keep;
            if (again) {
              const uint32_t nan = (kv_nan_bytes(w[y][j]) >> 7) * 0xffu;
              w[y][j] &= ~nan;
              if (nan) lds.found = 1;
            }
          }
        }
#pragma unroll
      for (int j = 0; j < 2 * DP; ++j) o[j] = mfma32<ACT>(kv_operand<ACT>(w[0][j], w[1][j], vs[h], vs[h]), p[h], o[j]);
    }
    if (__builtin_expect(ref.at != before, 0)) {
      place(at_hand);
      place(behind);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  if (tid == 0) lds.odd = lds.found = 0;
  for (;;) {
    m = KV_M_START;
    l = 0.f;
    ref = {0, KV_EXP_MIN};
#pragma unroll
    for (int d = 0; d < 2 * DP; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    ids = look_up(0);
    ids_next = look_up(1);
    look_up_scales(ids, at_hand);
    look_up_scales(ids_next, behind);
    __syncthreads();                       // (LDS is free)
    bring(0);
    bring(1);
    bring(2);
    settle(at_hand);
    settle(behind);
    for (int step = 0; step < steps; ++step) {
      // this tile has landed, the wave's pieces by its own count, the others' by the barrier; and everyone is done with the one
      // before, whose place the next but one takes
      vm_wait<2 * PER>();
      __syncthreads();
      bring(step + 3);
      const bool even = ((step >> 4) & 1) == 0;
      const int n = 4 * (step & 15);
      float ka[4], vs[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const auto pick = [&](float x, float y) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, even ? x : y), n + h)); };
        ka[h] = pick(at_hand.key, behind.key);
        vs[h] = pick(at_hand.value, behind.value);
      }
      const uint32_t wild = (uint32_t)((even ? at_hand.wild : behind.wild) >> n) & 15;
      const auto exponent = [&](int h) { return __builtin_amdgcn_readlane(even ? at_hand.exponent : behind.exponent, n + h); };
      if ((step & 15) == 4 && step > 15) {           // (the window before is done with: its place takes the one behind)
        if (even) ids_next = look_up((step >> 4) + 1);
        else ids = look_up((step >> 4) + 1);
      }
      if ((step & 15) == 9 && step > 15) {
        if (even) look_up_scales(ids_next, behind);
        else look_up_scales(ids, at_hand);
      }
      if ((step & 15) == 12 && step > 15) {
        if (even) settle(behind);
        else settle(at_hand);
      }
      // (waves whose rows see none of these keys, or that have no rows, only bring theirs)
      const int t0 = begin + MANY_STEP * step;
      if (!any_row || t0 > p_last || (a.window && t0 + MANY_STEP - 1 <= p_first - a.window)) continue;
      tile(step, ka, vs, wild, exponent);
    }
    vm_wait<0>();                          // (nothing may be on its way into LDS when the part ends)
    if (again) break;
    // 0 * NaN of a value that other rows see has reached rows that do not: then a second pass
    float any = 0.f;
#pragma unroll
    for (int d = 0; d < 2 * DP; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) any = __builtin_fmaf(o[d][e], 0.f, any);
    if (any != any && first + c32 < req.rows) lds.odd = 1;
    __syncthreads();
    if (!lds.odd) break;
    again = true;
  }
  __syncthreads();
  if (lds.found) {
    // the rows that do see a value that is no number: every dim of every key of the part is looked at
    for (int key = begin; key < end; ++key) {
      const int id = a.table[(size_t)pc.r * a.width + (key >> cache.block_shift)];
      if (id < 0 || id >= cache.n_blocks || key > p_row || (a.window && key <= p_row - a.window)) continue;
      const uint8_t* const page = cache.codes[1] + cache.page(id, pc.head);
#pragma unroll
      for (int j = 0; j < 2 * DP; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = 8 * (e >> 2) + 4 * hf + (e & 3), dim = DP == 2 ? (r & 15) + 16 * j + 64 * (r >> 4) : (r & 15) + 16 * j + 32 * (r >> 4);
          if ((page[kv_value_byte(key & ((1 << cache.block_shift) - 1), dim, cache.dim_shift)] & 0x7f) == 0x7f) o[j][e] = NAN;
        }
    }
  }

  const int at = 32 * wave + c32, row = row0 + at;
  const bool live = at < rows;
  float sum = l + __shfl_xor(l, 32, 64);
  if (pc.parts > 1) {
    // A partial result, in the order of the registers, so that a wave's stores lie side by side; the unit's last workgroup adds
    // all in order, each lane its own (by rows, a wave's loads 512 bytes apart: 64 tokens on 8000 124 us, 38 so and in shares of 8 steps)
    constexpr int STRIDE = R * (D + 2);
    float* const slot = crew.slots + (size_t)pc.slot * STRIDE;
    const float inv = (sum != 0.f ? 1.f / sum : 0.f) * kv_pow2(ref.at);
#pragma unroll
    for (int j = 0; j < 2 * DP; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        store16_device(slot + ((wave * 2 * DP + j) * 4 + e / 4) * 256 + 4 * lane,
                       __builtin_bit_cast(u32x4_t, float4_t{o[j][e], o[j][e + 1], o[j][e + 2], o[j][e + 3]} * inv));
    if (hf == 0) {
      kv_store_device(slot + R * D + at, m);
      kv_store_device(slot + R * (D + 1) + at, sum * KV_L_UNIT);
    }
    if (!kv_arrive(crew, pc, &lds.arrived)) return;
    const __amdgpu_buffer_rsrc_t slots = __builtin_amdgcn_make_buffer_rsrc((void*)crew.slots, 0, 3 * crew.shares * STRIDE * 4, 0x00020000);
    m = KV_M_START;
    sum = 0.f;
    ref.at = 0;                            // (partial results are numbers)
#pragma unroll
    for (int j = 0; j < 2 * DP; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][e] = 0.f;
    for (int k = 0; k < pc.parts; ++k) {
      const uint32_t from = (uint32_t)(pc.first_slot + k) * STRIDE;
      float4_t x[2 * DP][4];
#pragma unroll
      for (int j = 0; j < 2 * DP; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = kv_load4_device(slots, (from + ((wave * 2 * DP + j) * 4 + e) * 256 + 4 * lane) * 4);
      const float M = kv_load_device(crew.slots + from + R * D + at), L = kv_load_device(crew.slots + from + R * (D + 1) + at);
      const float most = fmaxf(m, M), f = __builtin_amdgcn_exp2f(m - most), w = L * __builtin_amdgcn_exp2f(M - most);
      m = most;
      sum = __builtin_fmaf(sum, f, w);
#pragma unroll
      for (int j = 0; j < 2 * DP; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[j][e] = __builtin_fmaf(o[j][e], f, x[j][e >> 2][e & 3] * w);
    }
  }
  const float inv = kv_inverse(sum, a, req, pc.r, row) * kv_pow2(ref.at);
  const int i = row / a.group;
  uint16_t* const to = a.out + (size_t)(req.start + i) * a.ldo + ((size_t)pc.head * a.group + (row - i * a.group)) * D;
#pragma unroll
  for (int j = 0; j < 2 * DP; ++j)
#pragma unroll
    for (int e = 0; e < 16; e += 8) {
      // elements e .. e + 3 are dims base + 4 hf .. + 4, the next four 8 further; lanes 32 apart exchange halves: eight dims in
      // a row each
      const int base = 16 * j + (DP == 2 ? 64 : 32) * (e >> 3);
      const float4_t x = float4_t{o[j][e], o[j][e + 1], o[j][e + 2], o[j][e + 3]} * inv;
      const float4_t y = float4_t{o[j][e + 4], o[j][e + 5], o[j][e + 6], o[j][e + 7]} * inv;
      const auto lo = __builtin_amdgcn_permlane32_swap(kv_pack<ACT>(x[0], x[1]), kv_pack<ACT>(y[0], y[1]), false, false);
      const auto hi = __builtin_amdgcn_permlane32_swap(kv_pack<ACT>(x[2], x[3]), kv_pack<ACT>(y[2], y[3]), false, false);
      if (live) *(u32x4_t*)(to + base + 8 * hf) = u32x4_t{lo[0], hi[0], lo[1], hi[1]};
    }
}

template <int ACT, int DP>
__device__ inline void kv_many(const AttendArgs& a, const KvCrew& crew, int wg, ManyLds<DP>& lds) {
  KvRequest req;
  long long all, total;
  const KvPart pc = kv_cut<MANY_ROWS, MANY_STEP>(a, crew, wg, req, all, total);
  if (pc.r >= 0) kv_many_part<ACT, DP>(a, crew, pc, req, lds);
}

}  // namespace glowq
