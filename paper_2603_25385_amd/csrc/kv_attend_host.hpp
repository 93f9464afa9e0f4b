// Launch of the attention kernels (internal).
#pragma once
#include "kv_attend.hpp"
#include "kv_host.hpp"

namespace glowq {

// rows of a workgroup's tile and keys of a step, for requests of few rows and of many
constexpr int KV_FEW_ROWS = 16, KV_FEW_STEP = 128, KV_MANY_ROWS = 128, KV_MANY_STEP = 64;
// n_many, n_few: workgroups of either kind
hipError_t launch_kv_attend(const AttendArgs& a, const KvCrew& many, const KvCrew& few, int n_many, int n_few, int act, hipStream_t st);

}  // namespace glowq
