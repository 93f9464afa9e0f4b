// Device-side building blocks of the latent cache.
//
// Token by token, in order of slots: latent_dim E4M3 codes, one scale byte, value = code * 2^(byte - 127), and rope_dim
// numbers of the activation type.  A scale of its own for every token: a token is written once and never moved to another grid.
#pragma once
#include "kv_device.hpp"

namespace glowq {

struct LatentView {
  uint8_t* codes;              // [n_blocks * block_tokens][latent_dim]
  uint8_t* scales;             // [n_blocks * block_tokens]
  uint16_t* ropes;             // [n_blocks * block_tokens][rope_dim]
  int n_blocks, block_shift;
  __device__ inline bool has(int slot) const { return slot >= 0 && slot >> block_shift < n_blocks; }
};

// Every value is a number of the cache's type: for binary16 none lies below its smallest, and none above MOST, the largest code value
// that the type holds: 240 * 2^8, of bfloat16 240 * 2^120 (the code behind 240 stands for 256, which is 2^16 and 2^128).
template <int ACT> struct LatentRange {
  static constexpr int LOW = ACT == ACT_F16 ? -15 : KV_EXP_MIN;
  static constexpr float MOST = ACT == ACT_F16 ? 61440.f : 0x1.ep127f;
};

}  // namespace glowq
