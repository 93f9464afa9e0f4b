// Host side of the cache operators (internal).
#pragma once
#include <hip/hip_runtime.h>
#include "../../include/glowq.h"
#include "kv_device.hpp"
#include "launch.hpp"

namespace glowq {

inline int kv_shift(int power_of_two) { return __builtin_ctz((unsigned)power_of_two); }
inline KvView kv_view(const glowq_kv_cache& c) {
  return KvView{{(uint8_t*)c.k_codes, (uint8_t*)c.v_codes}, {c.k_scales, c.v_scales}, c.n_blocks, c.kv_heads, kv_shift(c.block_tokens), kv_shift(c.head_dim)};
}
glowq_status kv_check_cache(const glowq_kv_cache* c, bool ptrs);

}  // namespace glowq
