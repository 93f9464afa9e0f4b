// Host side of the latent cache (internal).
#pragma once
#include "kv_host.hpp"
#include "latent_device.hpp"

namespace glowq {

inline LatentView latent_view(const glowq_latent_cache& c) {
  return LatentView{(uint8_t*)c.codes, c.scales, (uint16_t*)c.ropes, c.n_blocks, kv_shift(c.block_tokens)};
}
glowq_status latent_check_cache(const glowq_latent_cache* c, bool ptrs);

}  // namespace glowq
