// New tokens into the 8-bit cache of keys and values, run by run (device side).
#pragma once
#include "kv_device.hpp"

namespace glowq {

// Runs.  A run is a stretch of rows whose slots follow each other within one block.  A wave takes the runs that begin in its
// `per` rows, one after another, for one head's keys or values, and shares nothing with other waves.  Few rows: one for a wave,
// so that single tokens do not queue up; many: eight, since most rows begin nothing.
constexpr int RUN_THREADS = 256, RUN_WAVES = RUN_THREADS / 64;

inline int rows_per_wave(long long rows, int kv_heads) { return rows * 2 * kv_heads <= 32768 ? 1 : 8; }

// run(row, slot, tokens) for every run that begins in the wave's rows, none(row) for rows without a slot in the cache
template <class Run, class None>
__device__ inline void kv_runs(const KvView& c, const int32_t* slots, int T, int per, Run run, None none) {
  const int lane = threadIdx.x & 63, B = 1 << c.block_shift;
  const int row0 = blockIdx.x * per, row = row0 + lane;
  int s = -1, before = -2;
  if (lane < per && row < T) {
    s = slots[row];
    if (row > 0) before = slots[row - 1];
  }
  const bool here = lane < per && row < T, valid = s >= 0 && s >> c.block_shift < c.n_blocks;
  unsigned long long starts = __ballot(here && valid && !((s & (B - 1)) != 0 && before == s - 1));
  for (unsigned long long empty = __ballot(here && !valid); empty; empty &= empty - 1) none(row0 + __builtin_ctzll(empty));
  for (; starts; starts &= starts - 1) {
    const int at = __builtin_ctzll(starts), first = row0 + at, slot = __builtin_amdgcn_readlane(s, at);
    const int most = min(B - (slot & (B - 1)), T - first);
    int m = 0;
    for (; m < most; m += 64) {            // (128 tokens at most)
      const unsigned long long on = __ballot(m + lane < most && slots[min(first + m + lane, T - 1)] == slot + m + lane);
      if (~on) {
        m += __builtin_ctzll(~on);
        break;
      }
    }
    run(first, slot, min(m, most));
  }
}

// orders a wave's own LDS accesses across its lanes
__device__ inline void kv_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int ACT> __device__ inline uint32_t kv_encode_pair2(uint32_t lo, uint32_t hi, float scale) {
  typedef short short2_t __attribute__((ext_vector_type(2)));
  short2_t w = {0, 0};
  if constexpr (ACT == ACT_F16) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(half2_t, lo), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(half2_t, hi), scale, true);
  } else {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, lo), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, hi), scale, true);
  }
  return __builtin_bit_cast(uint32_t, w);
}

// A run of new tokens, rows first .. first + m of src (ld elements apart) at slots slot .., of one head's keys (which 0) or values
// (which 1).  image: of whole tiles of TOKENS tokens, in LDS, the wave's own, for values.
template <int ACT, int DP, int TOKENS>
__device__ inline void kv_append_run(const KvView& c, int which, int head, const uint16_t* src, long long ld, u32x4_t* image, int first, int slot, int m) {
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  constexpr int D = 64 * DP, PER_ROW = D / 16, TILE = 16 * D, LOADS = TOKENS * PER_ROW / 64;
  constexpr uint32_t INF = ACT == ACT_F16 ? 0x7c00u : 0x7f80u;
  const int lane = threadIdx.x & 63, B = 1 << c.block_shift;
  const int d = lane % PER_ROW * 16, token = lane / PER_ROW;
  const int block = slot >> c.block_shift, off = slot & (B - 1), end = off + m;
  uint8_t* const scale = c.scales[which] + (size_t)block * c.kv_heads + head;
  uint8_t* const page = c.codes[which] + c.page(block, head);
  const int byte = *scale;
  u32x4_t x[LOADS][2];
  // tokens from .. to of the block, in registers: zeros where there are none
  const auto load = [&](int from, int to) {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int t = from + token + k * (64 / PER_ROW);
      x[k][0] = x[k][1] = u32x4_t{0, 0, 0, 0};
      if (t < to) {
        const u32x4_t* p = (const u32x4_t*)(src + (size_t)(first + t - off) * ld + d);
        x[k][0] = p[0];
        x[k][1] = p[1];
      }
    }
  };
  // the run's largest finite magnitude, by its bits (those of 16 bits order as the numbers do)
  uint32_t top = 0;
  const auto most = [&] {
    u16x2_t mm = {0, 0};
#pragma unroll
    for (int k = 0; k < LOADS; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) mm = __builtin_elementwise_max(mm, __builtin_bit_cast(u16x2_t, x[k][i >> 2][i & 3] & 0x7fff7fffu));
    uint32_t h = max((uint32_t)mm[0], (uint32_t)mm[1]);
    if (__any(h >= INF)) {               // something that is no number: it does not count
      h = 0;
#pragma unroll
      for (int k = 0; k < LOADS; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t v = x[k][i >> 3][(i >> 1) & 3] >> (16 * (i & 1)) & 0x7fffu;
          h = v < INF ? max(h, v) : h;
        }
    }
    top = max(top, __builtin_bit_cast(uint32_t, kv_act_f32<ACT>(h)));
  };
  // whole tiles at a time but for the first
  const auto stretch = [&](int from) { return min(end, (from & ~15) + TOKENS); };
  for (int from = off; from < end; from = stretch(from)) {
    load(from, stretch(from));
    most();
  }
  for (int k = 1; k < 64; k <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, k, 64));
  const int before = off > 0 ? min(byte - 127, 126) : KV_EXP_MIN;
  const int e = max(before, kv_exponent(top));
  const float grid = kv_pow2(e), shrink = kv_pow2(max(before - e, -126));
  const bool grown = off > 0 && e > before, once = stretch(off) == end;
  if (lane == 0 && (off == 0 || grown)) *scale = (uint8_t)(e + 127);

  if (grown)                             // older tokens of the block to the new grid, values of the last tile below
    for (int u = lane; u < (which ? off >> 4 : (off + 15) >> 4) * (TILE / 16); u += 64) {
      if (!which && u / (TILE / 16) * 16 + (u & 15) >= off) continue;
      u32x4_t w = ((u32x4_t*)page)[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = kv_recode4(w[i], shrink);
      ((u32x4_t*)page)[u] = w;
    }
  for (int from = off; from < end; from = stretch(from)) {
    const int to = stretch(from), tile = from >> 4;
    if (!once) load(from, to);
    if (which) {
      kv_wave_sync();                    // (the stretch before has left)
      for (int u = lane; u < TILE / 16; u += 64) {
        u32x4_t w = {0, 0, 0, 0};
        const int t0 = tile * 16 + (u >> 4 & 3) * 4, older = min(4, off - t0);       // of the four tokens
        if (older > 0) {
          w = ((const u32x4_t*)page)[tile * (TILE / 16) + u];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (grown ? kv_recode4(w[i], shrink) : w[i]) & 0xffffffffu >> (8 * (4 - older));
        }
        image[u] = w;
      }
      for (int u = TILE / 16 + lane; u < ((to + 15 >> 4) - tile) * (TILE / 16); u += 64) image[u] = u32x4_t{0, 0, 0, 0};
      kv_wave_sync();
    }
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int t = from + token + k * (64 / PER_ROW);
      if (t >= to) continue;
      u32x4_t code;
#pragma unroll
      for (int i = 0; i < 4; ++i) code[i] = kv_encode_pair2<ACT>(x[k][i >> 1][(i & 1) * 2], x[k][i >> 1][(i & 1) * 2 + 1], grid);
      if (!which) *(u32x4_t*)(page + kv_key_byte(t, d, 6 + (DP == 2))) = code;
      else {
        uint8_t* const b = (uint8_t*)image + kv_value_byte(t - tile * 16, d, 6 + (DP == 2));
#pragma unroll
        for (int i = 0; i < 16; ++i) b[16 * i] = (uint8_t)(code[i >> 2] >> (8 * (i & 3)));
      }
    }
    if (which) {
      kv_wave_sync();
      for (int u = lane; u < ((to + 15 >> 4) - tile) * (TILE / 16); u += 64) ((u32x4_t*)page)[tile * (TILE / 16) + u] = image[u];
    }
  }
}

}  // namespace glowq
