// Launches of the attention kernels (internal).
#pragma once
#include "kv_attend.hpp"
#include "kv_host.hpp"

namespace glowq {

hipError_t launch_kv_attend_few(const AttendArgs& a, int act, int blocks_of_rows, int grid, hipStream_t st);

}  // namespace glowq
