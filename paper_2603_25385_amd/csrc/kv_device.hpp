// Device-side building blocks of the 8-bit cache of keys and values: its layout, its codes.
//
// A block of `block_tokens` tokens of one key/value head is a page of block_tokens * head_dim E4M3 codes and one scale
// byte, value = code * 2^(byte - 127).  Pages are arrays of 16-token tiles, a tile of one 1 KiB piece per 64 dims, a piece
// [64 lanes][16 bytes]: what one wave loads at once and what the attention kernels' matrix instructions take as it stands.
//   keys    lane 16 g + t: token t, dims 16 g .. + 16 of the piece     (contraction over dims: 8 consecutive per lane)
//   values  lane 16 g + d: tokens 4 g .. + 4 of dim d + 16 j in word j (contraction over tokens: 4 consecutive per word)
#pragma once
#include "common.hpp"

namespace glowq {

constexpr int KV_PIECE = 1024;       // bytes: 16 tokens x 64 dims
constexpr int KV_EXP_MIN = -64;      // exponent of a block's scale at least; smallest value 2^-73
constexpr uint32_t KV_MAX_CODE = 0x43e00000u;      // 448.0f, the largest E4M3 magnitude

// the cache as the kernels see it
struct KvView {
  uint8_t* codes[2];           // keys, values: [n_blocks][kv_heads][page]
  uint8_t* scales[2];          // [n_blocks][kv_heads]
  int n_blocks, kv_heads;
  int block_shift;             // log2(block_tokens)
  int dim_shift;               // log2(head_dim)
  __device__ inline size_t page(int block, int head) const { return ((size_t)block * kv_heads + head) << (block_shift + dim_shift); }
};

// byte of (token, dim) in a page
__device__ inline int kv_key_byte(int t, int d, int dim_shift) {
  return (((t >> 4) << (dim_shift - 6)) + (d >> 6)) * KV_PIECE + ((((d >> 4) & 3) << 4) + (t & 15)) * 16 + (d & 15);
}
__device__ inline int kv_value_byte(int t, int d, int dim_shift) {
  return (((t >> 4) << (dim_shift - 6)) + (d >> 6)) * KV_PIECE + ((((t >> 2) & 3) << 4) + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (t & 3);
}

template <int ACT> __device__ inline float kv_act_f32(uint32_t h) {
  if constexpr (ACT == ACT_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
  else return __builtin_bit_cast(float, h << 16);
}

// The exponent of a block whose largest finite magnitude has this fp32 pattern: the smallest e with max <= 448 * 2^e.
// (448 = 1.75 * 2^8, so the fraction decides between the maximum's own exponent less 8 and one more.)
__device__ inline int kv_exponent(uint32_t top) {
  const int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > (KV_MAX_CODE & 0x7fffffu));
  return max(e, KV_EXP_MIN);
}

// 2^e, -126 <= e <= 127
__device__ inline float kv_pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// Four values, already divided by the block's scale, as E4M3 codes: nearest even; what is not finite becomes the NaN code.
__device__ inline uint32_t kv_encode4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  uint32_t r = (uint32_t)w;
  const auto odd = [](float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) == 0x7f800000u; };
  if (odd(a)) r |= 0x7fu;
  if (odd(b)) r |= 0x7f00u;
  if (odd(c)) r |= 0x7f0000u;
  if (odd(d)) r |= 0x7f000000u;
  return r;
}

// Four codes moved to the grid of a scale 2^down times as large, nearest even.
__device__ inline uint32_t kv_recode4(uint32_t w, float shrink) {
  typedef float float2_t __attribute__((ext_vector_type(2)));
  const float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return kv_encode4(lo[0] * shrink, lo[1] * shrink, hi[0] * shrink, hi[1] * shrink);
}

}  // namespace glowq
