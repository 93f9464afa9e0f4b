// Attention over the 8-bit cache for few rows per (request, key/value head): single tokens.
//
// A wave reads keys and values straight into its registers, 32 tokens at a time, the next 32 on their way: no byte is needed by
// two waves.  Scores come transposed, S^T = K Q^T (16x16x32), so that a lane holds four keys of one row: the row's largest score
// is looked for across lanes only when it has outgrown the reference, and the weights are the second product's operand,
// O^T = V^T P^T, as they stand.  The waves' results meet in LDS.
#pragma once
#include <type_traits>
#include "kv_attend.hpp"

namespace glowq {

constexpr int FEW_THREADS = 256, FEW_WAVES = FEW_THREADS / 64, FEW_ROWS = 16;
constexpr int FEW_KEYS = 32;                          // of a wave's tile
constexpr int FEW_STEP = FEW_KEYS * FEW_WAVES;

// Keys and values of 32 tokens as they lie in the cache: [16-token tile][64 dims]
template <int DP> struct KvTile {
  u32x4_t k[2][DP], v[2][DP];
};

template <int DP> struct FewLds {
  union {
    float o[2][FEW_ROWS][64 * DP + 4];                // (rows 16 bytes apart in their banks)
    float join[FEW_THREADS * 10];
  };
  float m[FEW_WAVES][FEW_ROWS], l[FEW_WAVES][FEW_ROWS];
  int at[FEW_WAVES];
  uint32_t arrived;
};

// PAST: codes are loaded past the last-level cache (see kv_few)
template <int ACT, int DP, bool PAST>
__device__ inline void kv_few_part(const AttendArgs& a, const KvCrew& crew, const KvPart& pc, const KvRequest& req, FewLds<DP>& lds) {
  constexpr int R = FEW_ROWS, D = 64 * DP;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g = lane >> 4;
  const KvView& cache = a.cache;

  // keys and rows
  const int rows = req.rows, i1 = __builtin_amdgcn_readfirstlane((rows - 1) / a.group);
  const int begin = req.lo(0, a.window) + pc.first * FEW_STEP, end = min(req.hi(i1), begin + pc.count * FEW_STEP);
  const int p_first = req.p0, p_last = req.p0 + i1, p_row = req.p0 + c16 / a.group;
  const int tiles = end > begin ? (end - begin + FEW_KEYS - 1) / FEW_KEYS : 0;        // of all waves
  const int mine = tiles > wave ? (tiles - wave + FEW_WAVES - 1) / FEW_WAVES : 0;

  // where 32 of the wave's tiles lie, two tiles, the rows' queries
  u32x4_t q[DP][2];
  uint32_t at_lo, at_hi;
  float key_scale, value_scale;
  int value_exponent, bytes[2];
  bool there;
  unsigned long long absent, wild;     // lanes whose tile is not there, whose values need more than their scale
  KvReference ref = {0, KV_EXP_MIN};
  KvTile<DP> t[2];
  const auto place = [&] {
    value_scale = kv_value_scale(value_exponent, ref.at);
    wild = __ballot(kv_wild<ACT>(value_exponent, ref.at));
  };
  const auto look_up = [&](int k0) {
    // lane 2 k + s: where 16-token tile s of this wave's tile k0 + k lies, and its scales.  Tiles that no row sees count as not
    // there: nobody need have written their block, nor the one whose bytes are read in place of what is not there
    const int token = begin + (wave + FEW_WAVES * (k0 + (lane >> 1))) * FEW_KEYS + 16 * (lane & 1);
    const bool seen = token < end && (!a.window || token + 15 > p_first - a.window);
    int id = seen ? a.table[(size_t)pc.r * a.width + (token >> cache.block_shift)] : -1;
    const bool ok = id >= 0 && id < cache.n_blocks;
    if (!ok) id = 0;
    const size_t at = cache.page(id, pc.head) + (ok ? (size_t)((token & ((1 << cache.block_shift) - 1)) >> 4) * DP * KV_PIECE : 0);
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
    const size_t sc = (size_t)id * cache.kv_heads + pc.head;
    bytes[0] = cache.scales[0][sc];
    bytes[1] = cache.scales[1][sc];
    there = ok;
  };
  // (once the first tiles are on their way: it waits for the bytes)
  const auto settle = [&] {
    const int e = bytes[1] - 127;
    key_scale = there ? kv_pow2(bytes[0] - 127) * a.scale : 1.f;
    value_exponent = !there ? KV_ABSENT : e < KvRange<ACT>::ZERO ? KV_ZEROS : e;
    absent = __ballot(!there);
    place();
  };
  const auto fetch = [&](int k, KvTile<DP>& x) {
    k = min(k, 31);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const size_t off = (size_t)(uint32_t)__builtin_amdgcn_readlane(at_lo, 2 * k + s) | (size_t)(uint32_t)__builtin_amdgcn_readlane(at_hi, 2 * k + s) << 32;
      const u32x4_t* kp = (const u32x4_t*)(cache.codes[0] + off);
      const u32x4_t* vp = (const u32x4_t*)(cache.codes[1] + off);
#pragma unroll
      for (int d = 0; d < DP; ++d) {
        x.k[s][d] = PAST ? __builtin_nontemporal_load(kp + 64 * d + lane) : kp[64 * d + lane];
        x.v[s][d] = PAST ? __builtin_nontemporal_load(vp + 64 * d + lane) : vp[64 * d + lane];
      }
    }
  };
  look_up(0);
  {
    const bool live = c16 < rows;
    const int i = live ? c16 / a.group : 0;
    const uint16_t* src = a.q + (size_t)(req.start + i) * a.ldq + ((size_t)pc.head * a.group + (live ? c16 - i * a.group : 0)) * D + 16 * g;
#pragma unroll
    for (int d = 0; d < DP; ++d)
#pragma unroll
      for (int h = 0; h < 2; ++h) q[d][h] = *(const u32x4_t*)(src + 64 * d + 8 * h);
  }
  fetch(0, t[0]);
  fetch(1, t[1]);
  settle();

  float4_t o[DP * 4];
  float m = KV_M_START, l = 0.f;
  bool odd = false;                    // tiles were put off: see `run`
#pragma unroll
  for (int d = 0; d < DP * 4; ++d) o[d] = float4_t{0.f, 0.f, 0.f, 0.f};
  const auto pass = [&](const auto again) {
    for (int k0 = 0; k0 < mine; k0 += 32) {
      if (again.value || k0 > 0) {
        look_up(k0);
        fetch(0, t[0]);
        fetch(1, t[1]);
        settle();
      }
      const auto run = [&](int k, KvTile<DP>& x) __attribute__((always_inline)) {
        const int t0 = begin + (wave + FEW_WAVES * (k0 + k)) * FEW_KEYS;
        const uint32_t gone = (uint32_t)(absent >> 2 * k) & 3, wilds = (uint32_t)(wild >> 2 * k) & 3;
        const auto pick = [&](float v, int h) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 2 * k + h)); };
        float ka[2] = {pick(key_scale, 0), pick(key_scale, 1)};
        float4_t s[2] = {float4_t{0.f, 0.f, 0.f, 0.f}, float4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int d = 0; d < DP; ++d)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[h] = mfma16<ACT>(kv_operand<ACT>(x.k[h][d][2 * u], x.k[h][d][2 * u + 1]), q[d][u], s[h]);
        if (!(!gone && t0 + FEW_KEYS - 1 <= p_first && t0 + FEW_KEYS <= end && (!a.window || t0 > p_last - a.window))) {
          // Hidden keys have no score, and what lies behind the last token may be anything.  0 * NaN must not reach rows that do
          // not see the NaN: a tile with such values is put off to a second pass, which takes zeros for them
          const int most = min(end - 1, p_row), least = a.window ? p_row - a.window : -1;
          uint32_t nan_bytes = 0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int key = t0 + 16 * h + 4 * g;
            const bool ok = !(gone >> h & 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[h][e] = ok && key + e <= most && key + e > least ? s[h][e] * ka[h] : -INFINITY;
#pragma unroll
            for (int d = 0; d < DP; ++d)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (!ok) x.v[h][d][j] = 0;
                const uint32_t n = kv_nan_bytes(x.v[h][d][j]);
                nan_bytes |= n;
                if constexpr (again.value) x.v[h][d][j] &= ~((n >> 7) * 0xffu);
              }
          }
          ka[0] = ka[1] = 1.f;           // (in the scores already: a scale may be 0 in fp32, and -inf times 0 is no number)
          const bool put_off = __any(nan_bytes != 0);
          if (again.value != put_off) {
            odd = true;
            return;
          }
        } else if (again.value) return;
        float most = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h) most = fmaxf(most, fmaxf(fmaxf(s[h][0], s[h][1]), fmaxf(s[h][2], s[h][3])) * ka[h]);
        if (__any(most > m + KV_M_SLACK)) {
          most = fmaxf(most, __shfl_xor(most, 16, 64));
          most = fmaxf(fmaxf(most, __shfl_xor(most, 32, 64)), m);
          const float f = __builtin_amdgcn_exp2f(m - most);
          m = most;
          l *= f;
#pragma unroll
          for (int d = 0; d < DP * 4; ++d) o[d] *= f;
        }
        __builtin_amdgcn_sched_barrier(0);     // (conversions of the values stay behind it: registers)
        u32x4_t p;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][i], ka[h], -m));
          p[2 * h] = kv_pack<ACT>(e[0], e[1]);
          p[2 * h + 1] = kv_pack<ACT>(e[2], e[3]);
          l = kv_add2<ACT>(p[2 * h + 1], kv_add2<ACT>(p[2 * h], l));
        }
        __builtin_amdgcn_sched_barrier(0);
        float vs[2] = {pick(value_scale, 0), pick(value_scale, 1)};
        uint32_t todo = 3;
        do {
          uint32_t set = 3;
          u32x4_t w = p;
          if (__builtin_expect(wilds != 0, 0)) {
            // both halves in one product where their scales fit together, those of 2^-16 of the other in a second one
            const int before = ref.at;
            int ev[2], high = KV_ABSENT;
            bool need = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              ev[h] = __builtin_amdgcn_readlane(value_exponent, 2 * k + h);
              if (!(todo >> h & 1) || ev[h] <= KV_ZEROS) continue;
              high = max(high, ev[h]);
              need |= kv_wild<ACT>(ev[h], ref.at);
            }
            if (need)
              kv_refer(high, ref, [&](int by) {
#pragma unroll
                for (int d = 0; d < DP * 4; ++d)
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[d][e] = __builtin_ldexpf(o[d][e], by);
              });
            set = todo;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (need && ev[h] > KV_ZEROS && ev[h] < high && ev[h] - ref.at < KvRange<ACT>::LOW) set &= ~(1u << h);
              vs[h] = set >> h & 1 ? kv_value_scale(ev[h], ref.at) : 1.f;
              if (!(set >> h & 1)) w[2 * h] = w[2 * h + 1] = 0;
            }
            if (ref.at != before) place();
          }
#pragma unroll
          for (int d = 0; d < DP; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[4 * d + j] = mfma16<ACT>(kv_operand<ACT>(x.v[0][d][j], x.v[1][d][j], vs[0], vs[1]), w, o[4 * d + j]);
          todo &= ~set;
        } while (todo);
      };
      const int here = min(32, mine - k0);
      for (int k = 0; k < here; k += 2) {
        run(k, t[0]);
        fetch(k + 2, t[0]);
        if (k + 1 < here) run(k + 1, t[1]);
        fetch(k + 3, t[1]);
      }
    }
  };
  pass(std::false_type{});
  if (odd) {
    pass(std::true_type{});
    // the rows that do see such a value get theirs: every dim of every key of the part is looked at again (by each wave: what
    // one marks stays marked in the sum)
    for (int key = begin; key < end; ++key) {
      const int id = a.table[(size_t)pc.r * a.width + (key >> cache.block_shift)];
      if (id < 0 || id >= cache.n_blocks || key > p_row || (a.window && key <= p_row - a.window)) continue;
      const uint8_t* const page = cache.codes[1] + cache.page(id, pc.head);
#pragma unroll
      for (int d = 0; d < DP * 4; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((page[kv_value_byte(key & ((1 << cache.block_shift) - 1), 16 * d + 4 * g + e, cache.dim_shift)] & 0x7f) == 0x7f) o[d][e] = NAN;
    }
  }

  // the waves' results become one: the rows' largest reference and the waves' largest exponent, then sums of two waves each through LDS
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) {
    lds.m[wave][c16] = m;
    lds.l[wave][c16] = l;
  }
  if (lane == 0) lds.at[wave] = ref.at;
  __syncthreads();
  const int at = __builtin_amdgcn_readfirstlane(max(max(lds.at[0], lds.at[1]), max(lds.at[2], lds.at[3])));
  const float f = __builtin_amdgcn_exp2f(m - fmaxf(fmaxf(lds.m[0][c16], lds.m[1][c16]), fmaxf(lds.m[2][c16], lds.m[3][c16]))) * kv_pow2(max(ref.at - at, -126));
#pragma unroll
  for (int turn = 0; turn < 2; ++turn) {
    if ((wave >> 1) == 1 - turn)
#pragma unroll
      for (int d = 0; d < DP * 4; ++d) {
        float4_t* to = (float4_t*)&lds.o[wave & 1][c16][16 * d + 4 * g];
        const float4_t x = o[d] * f;
        *to = turn ? x + *to : x;
      }
    __syncthreads();
  }
  // rows out, or a partial result: eight dims a thread
  const bool split = pc.parts > 1;
  float* const slot = split ? crew.slots + (size_t)pc.slot * (R * (D + 2)) : nullptr;
  for (int u = tid; u < rows * (D / 8); u += FEW_THREADS) {
    const int row = u / (D / 8), d = u % (D / 8) * 8;
    const float top = fmaxf(fmaxf(lds.m[0][row], lds.m[1][row]), fmaxf(lds.m[2][row], lds.m[3][row]));
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) sum += lds.l[w][row] * __builtin_amdgcn_exp2f(lds.m[w][row] - top);
    float x[8];
    const float inv = (!split ? kv_inverse(sum, a, req, pc.r, row) : sum != 0.f ? 1.f / sum : 0.f) * kv_pow2(at);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (lds.o[0][row][d + e] + lds.o[1][row][d + e]) * inv;
    if (!split) kv_store_row<ACT, D>(a, req, pc.head, row, d, x);
    else {
#pragma unroll
      for (int e = 0; e < 8; e += 4) store16_device(slot + row * D + d + e, __builtin_bit_cast(u32x4_t, float4_t{x[e], x[e + 1], x[e + 2], x[e + 3]}));
      if (d == 0) {
        kv_store_device(slot + R * D + row, top);
        kv_store_device(slot + R * (D + 1) + row, sum * KV_L_UNIT);
      }
    }
  }
  if (split && kv_arrive(crew, pc, &lds.arrived)) kv_join<ACT, D, R, FEW_THREADS>(a, crew, req, pc, 0, rows, lds.join);
}

// Calls that read more than half of the last-level cache (256 MB) go past it: 64 requests at ragged lengths up to 8000 (578 MB)
// 114 -> 104 us, 5.5 TB/s; smaller ones may find there what an earlier call left: 32 requests up to 2000 (75 MB) would take 21.0
// instead of 19.6 in a loop over three caches.
template <int ACT, int DP>
__device__ inline void kv_few(const AttendArgs& a, const KvCrew& crew, int wg, FewLds<DP>& lds) {
  KvRequest req;
  long long all, total;
  const KvPart pc = kv_cut<FEW_ROWS, FEW_STEP>(a, crew, wg, req, all, total);
  if (pc.r < 0) return;
  if (all * (FEW_STEP * 2 * 64 * DP) > (128ll << 20)) kv_few_part<ACT, DP, true>(a, crew, pc, req, lds);
  else kv_few_part<ACT, DP, false>(a, crew, pc, req, lds);
}

}  // namespace glowq
