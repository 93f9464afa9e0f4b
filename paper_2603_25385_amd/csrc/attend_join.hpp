// The second launch of attention whose units were cut: rows from their partial results.
#pragma once
#include "kv_attend.hpp"

namespace glowq {

constexpr int JOIN_THREADS = 256;

// Workgroups of a partial result's place, so that a grid has some 2000 where there is that much to do: `slots` at most
inline int join_split(int slots) { return slots >= 1024 ? 1 : slots >= 512 ? 2 : slots >= 256 ? 4 : 8; }

// What the first launch leaves for the second in the workspace, one for every place of a partial result: the part that left it.  (The
// second finding all parts again, as the first does, took 3 us of its 10.)
struct JoinTicket {
  int r, head, tile, parts, first_slot, slot;              // r < 0: no partial result here
  int start, fresh, rows, p0, len;
  int unused[5];
};

// slots: places, no more than workgroups; those behind the partial results that there are say so, each through the workgroup of its number
__device__ inline void join_leave(JoinTicket* tickets, int slots, const KvPart& pc, const KvRequest& req) {
  if (threadIdx.x) return;
  if (pc.r >= 0 && pc.parts > 1)
    tickets[pc.slot] = {pc.r, pc.head, pc.tile, pc.parts, pc.first_slot, pc.slot, req.start, req.fresh, req.rows, req.p0, req.len, {}};
  if ((int)blockIdx.x >= pc.slots && (int)blockIdx.x < slots) tickets[blockIdx.x].r = -1;
}
// Whether there is something to join
__device__ inline bool join_take(const JoinTicket* tickets, KvPart& pc, KvRequest& req) {
  const JoinTicket t = tickets[blockIdx.x];
  if (t.r < 0) return false;
  pc = {t.r, t.head, t.tile, 0, 0, t.parts, t.first_slot, t.slot, 0};
  req.start = t.start;
  req.fresh = t.fresh;
  req.rows = t.rows;
  req.p0 = t.p0;
  req.len = t.len;
  return true;
}

// A partial result of R rows of D numbers: O, four numbers of a row together, in any order; then M of the rows, then l.
template <int R, int D> constexpr int join_stride() { return R * (D + 2); }

// out = sum f O / sum f l, f = 2^(M - max M), parts in order.  The workgroups of a part (gridDim.y of them) join an equal share of its
// unit's numbers, the first `items` fours, so that all of the machine reads (one: 24 us after 64 requests of 128 heads); where shares
// are short, groups of threads take every so many parts each.  place(item, row, dim): whose numbers the four at `item` are;
// inverse(l, row): 1 / l; row counted from the tile's first; store(row, dim, four numbers).
template <int R, int D, class Place, class Inverse, class Store>
__device__ inline void attend_join(const KvCrew& crew, const KvPart& pc, int rows, int items, float (*scratch)[6], Place place, Inverse inverse, Store store) {
  constexpr int STRIDE = join_stride<R, D>();
  const int k = (pc.slot - pc.first_slot) * gridDim.y + blockIdx.y, shares = pc.parts * gridDim.y;
  const int from = (int)((long long)items * k / shares), n = (int)((long long)items * (k + 1) / shares) - from;
  int lanes = JOIN_THREADS;                // to one group
  while (lanes > 16 && lanes / 2 >= n) lanes /= 2;
  const int groups = JOIN_THREADS / lanes, group = threadIdx.x / lanes;
  const float* const results = crew.slots + (size_t)pc.first_slot * STRIDE;
  for (int first = 0; first < n; first += lanes) {         // (as often for all threads)
    const int at = first + threadIdx.x % lanes, item = from + min(at, n - 1);
    int row, dim;
    place(item, row, dim);
    float top = KV_M_START, sum = 0.f;
    float4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = group; i < pc.parts; i += groups) {
      const float* const r = results + (size_t)i * STRIDE;
      const float M = r[R * D + row], l = r[R * (D + 1) + row];
      const float4_t o = *(const float4_t*)(r + 4 * item);
      const float most = fmaxf(top, M), f = __builtin_amdgcn_exp2f(top - most), w = __builtin_amdgcn_exp2f(M - most);
      top = most;
      sum = __builtin_fmaf(sum, f, l * w);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(x[e], f, o[e] * w);
    }
    if (groups > 1) {
      float* const mine = scratch[threadIdx.x];
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[e] = x[e];
      mine[4] = top;
      mine[5] = sum;
      __syncthreads();
      if (group == 0)
        for (int i = 1; i < groups; ++i) {
          const float* const other = scratch[threadIdx.x + i * lanes];
          const float most = fmaxf(top, other[4]), f = __builtin_amdgcn_exp2f(top - most), w = __builtin_amdgcn_exp2f(other[4] - most);
          top = most;
          sum = sum * f + other[5] * w;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = x[e] * f + other[e] * w;
        }
      __syncthreads();
    }
    if (group == 0 && at < n && row < rows) store(row, dim, x * inverse(sum, row));
  }
}

}  // namespace glowq
