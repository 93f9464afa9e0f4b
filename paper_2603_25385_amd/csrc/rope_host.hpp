// Host side of rotary positions (internal).
#pragma once
#include <hip/hip_runtime.h>
#include "../../include/glowq.h"
#include "launch.hpp"
#include "rope_device.hpp"

namespace glowq {

inline RopeView rope_view(const glowq_rope& r) {
  return RopeView{(const unsigned long long*)r.turns, r.rotary_dim / 16, r.layout == GLOWQ_ROPE_PAIRS, r.magnitude};
}
// head_dim: of the heads that it is for
glowq_status check_rope(const glowq_rope* rope, int head_dim);
// rows of heads of `dim` numbers, T of them
glowq_status check_rope_rows(const glowq_rope_rows* rows, int n_rows, int dim, int dtype);
long long rope_threads(const glowq_rope_rows* rows, int n_rows, int dim, int dtype, int T);
// threads: how many the call takes (T * groups * units)
RotateArgs make_rotate_args(const glowq_rope& rope, const glowq_rope_rows* rows, int n_rows, int dim, int dtype, const int32_t* positions, int T,
                            long long* threads);

}  // namespace glowq
