// Launches of the attention kernels (internal).
#pragma once
#include "kv_attend.hpp"
#include "kv_host.hpp"

namespace glowq {

constexpr int MANY_ROW_BLOCKS = 1, MANY_WAVES = 4, MANY_ROWS = 32 * MANY_ROW_BLOCKS * MANY_WAVES;
hipError_t launch_kv_attend_many(const AttendArgs& a, int act, int grid, hipStream_t st);
hipError_t launch_kv_attend_few(const AttendArgs& a, int act, int blocks_of_rows, int grid, hipStream_t st);

}  // namespace glowq
