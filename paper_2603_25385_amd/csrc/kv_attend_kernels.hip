// Attention over the 8-bit cache: its kernels.
#include "kv_attend_host.hpp"
#include "kv_few.hpp"
#include "kv_many.hpp"

namespace glowq {

static_assert(FEW_THREADS == MANY_THREADS, "one launch holds both kinds of workgroups");
static_assert(KV_FEW_ROWS == FEW_ROWS && KV_FEW_STEP == FEW_STEP && KV_MANY_ROWS == MANY_ROWS && KV_MANY_STEP == MANY_STEP, "sizes of workspace and grid");

// Single tokens and others of few rows alone.  (Heads of 128: two workgroups on a CU are enough to read with; 64 requests up to 8000
// tokens 105 us, 109 with the three that registers would allow.  Heads of 64, half the bytes in flight: four; 200 requests up to
// 1500, 8 heads, 46 us, 55 with two.)
template <int ACT, int DP>
__global__ void __launch_bounds__(FEW_THREADS) __attribute__((amdgpu_waves_per_eu(2, DP == 2 ? 2 : 4))) k_kv_attend_few(AttendArgs a, KvCrew few) {
  __shared__ FewLds<DP> lds;
  kv_few<ACT, DP>(a, few, blockIdx.x, lds);
}

// A request of many rows alone.  (Rows of 64 dims leave registers for three workgroups on a CU, rows of 128 for two.)
template <int ACT, int DP>
__global__ void __launch_bounds__(MANY_THREADS, 4 - DP) k_kv_attend_many(AttendArgs a, KvCrew many) {
  __shared__ ManyLds<DP> lds;
  kv_many<ACT, DP>(a, many, blockIdx.x, lds);
}

// Requests of many rows, and of few beside them: the first workgroups take the former.
template <int ACT, int DP>
__global__ void __launch_bounds__(MANY_THREADS, 4 - DP) k_kv_attend(AttendArgs a, KvCrew many, KvCrew few, int n_many) {
  __shared__ union { ManyLds<DP> many; FewLds<DP> few; } lds;
  if ((int)blockIdx.x < n_many) kv_many<ACT, DP>(a, many, blockIdx.x, lds.many);
  else kv_few<ACT, DP>(a, few, blockIdx.x - n_many, lds.few);
}

template <int ACT, int DP> static void go(const AttendArgs& a, const KvCrew& many, const KvCrew& few, int n_many, int n_few, hipStream_t st) {
  if (!n_many) k_kv_attend_few<ACT, DP><<<dim3(n_few), dim3(FEW_THREADS), 0, st>>>(a, few);
  else if (!n_few) k_kv_attend_many<ACT, DP><<<dim3(n_many), dim3(MANY_THREADS), 0, st>>>(a, many);
  else k_kv_attend<ACT, DP><<<dim3(n_many + n_few), dim3(MANY_THREADS), 0, st>>>(a, many, few, n_many);
}
hipError_t launch_kv_attend(const AttendArgs& a, const KvCrew& many, const KvCrew& few, int n_many, int n_few, int act, hipStream_t st) {
  if (a.cache.dim_shift == 6) act == GLOWQ_F16 ? go<ACT_F16, 1>(a, many, few, n_many, n_few, st) : go<ACT_BF16, 1>(a, many, few, n_many, n_few, st);
  else act == GLOWQ_F16 ? go<ACT_F16, 2>(a, many, few, n_many, n_few, st) : go<ACT_BF16, 2>(a, many, few, n_many, n_few, st);
  return hipGetLastError();
}

}  // namespace glowq
