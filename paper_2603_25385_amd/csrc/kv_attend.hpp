// Attention over the 8-bit cache: what its kernels share.
//
// Rows.  The `group` q heads of a key/value head and the new tokens of a request are one list of rows, row = token * group
// + head, so that everything that reads a head's keys shares what it has read.  A workgroup takes a tile of rows of one
// (request, key/value head) and a stretch of its keys, a piece.
//
// Shares.  Lengths are known on the GPU only, so the kernels share out the work themselves.  A unit is a tile of rows of one
// head of one request, a step a stretch of its keys.  All units' steps stand in a row, and every workgroup takes as many of
// them as the next, ceil(all / workgroups), whatever the lengths are: parts of two units at most, and whole ones between.
// A unit that one workgroup takes whole is stored directly; the parts of others leave partial results, and the workgroup that
// finds all others of its unit counted joins them in order.  (Where units are many, a workgroup takes one whole unit instead.)
//
// Scales.  Keys' and values' codes enter the matrix cores as they are.  A block's key scale is a factor of its scores, its
// value scale 2^e is added to the exponent: with t = score + e (base 2) and a reference M per row,
//     P = 2^(t - M),   O = sum P code,   l = sum 2^-e P,   out = O / l.
// M is the largest t so far or up to M_SLACK less: O and l are rescaled only when a row's t outgrows it by more.
#pragma once
#include "kv_device.hpp"

namespace glowq {

constexpr float KV_M_START = -1.7e38f;    // below every score; finite, so that 2^(-inf - M) is 0
constexpr float KV_M_SLACK = 8.f;         // P <= 2^8: far inside binary16
constexpr float KV_LOG2E = 1.4426950408889634f;

struct AttendArgs {
  KvView cache;
  const uint16_t* q;
  uint16_t* out;
  const int32_t *table, *lengths, *starts;
  long long ldq, ldo;
  int width, n, T, heads, group;
  int max_fresh, cap;            // bounds of a request: new tokens, keys
  int window;                    // 0: none
  float scale;                   // of the scores, times log2(e)
};

// Part of a kernel's workgroups, and what they need.
struct KvCrew {
  int rows_from, rows_to;        // it serves requests of rows_from < rows <= rows_to
  int workgroups;                // that share the steps
  int least;                     // steps of a share
  int whole;                     // a workgroup takes one unit, where units are short or many enough (the grid has enough then)
  uint32_t* counts;              // workspace: arrivals at units that are cut
  float* slots;                  // ... partial results, two per share
};

// What the kernels know of a request.
struct KvRequest {
  int start, fresh, rows, p0, len;
  KvRequest() = default;
  __device__ inline KvRequest(const AttendArgs& a, const KvCrew& crew, int r) {
    const int from = a.starts[r], to = a.starts[r + 1], length = max(a.lengths[r], 0);
    start = min(max(from, 0), a.T);
    fresh = min(min(max(to - start, 0), a.max_fresh), a.T - start);
    rows = fresh * a.group;
    if (rows <= crew.rows_from || rows > crew.rows_to) rows = 0;
    p0 = length - fresh;
    len = min(length, a.cap);
  }
  // keys [lo, hi) of new tokens i0 .. i1, lo at a 32-token boundary
  __device__ inline int hi(int i1) const { return max(0, min(len, p0 + i1 + 1)); }
  __device__ inline int lo(int i0, int window) const { return window ? max(0, p0 + i0 - window + 1) & ~31 : 0; }
  // ... in steps, one at least
  __device__ inline int steps(int i0, int i1, int window, int step) const {
    const int n = hi(i1) - lo(i0, window);
    return n > 0 ? (n + step - 1) / step : 1;
  }
};

// A workgroup's part of a unit: steps first .. first + count of `steps` (the unit's).  parts: workgroups that have a part of it,
// counted at word first_wg; slot: of the partial result, where there are several.
struct KvPart {
  int r, head, tile;             // r < 0: none (any more)
  int first, count, steps;
  int parts, first_wg, first_slot, slot;
};
struct KvShare {
  long long at, end;             // steps that are left to this workgroup, counted over all units
  long long all, per;            // steps of all units, of a share
  long long before, mine;        // steps of the requests before this thread's, and of its own
  int wg, whole;                 // one unit each, and steps are units
};
template <int THREADS> struct KvShareLds {
  long long sum[THREADS / 64];
  long long first;               // steps of the requests before
  int r, unit_steps;
  KvRequest q;
};

// v / by, both positive (the division of 64 bits takes five times as long)
__device__ inline long long kv_quotient(long long v, long long by) {
  return (v | by) >> 32 ? v / by : (long long)((uint32_t)v / (uint32_t)by);
}

__device__ inline long long kv_uniform(long long v) {
  return (long long)((unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) | (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}

// sum over the workgroup of v; `before`: over the threads before this one
template <int THREADS> __device__ inline long long kv_scan(long long v, long long* waves, long long& before) {
  long long s = v;
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(s, d, 64);
    if ((int)(threadIdx.x & 63) >= d) s += o;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  long long total = 0;
  before = s - v;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) before += waves[w];
    total += waves[w];
  }
  return kv_uniform(total);
}

// Units of a request, and the steps that each is taken to have (those of its last rows: the most)
template <int R> __device__ inline int kv_units(const KvRequest& q, int kv_heads) { return (q.rows + R - 1) / R * kv_heads; }
template <int STEP> __device__ inline int kv_unit_steps(const AttendArgs& a, const KvRequest& q) { return q.steps(0, q.fresh - 1, a.window, STEP); }

// The workgroup's share, wg of crew.workgroups.  Then, one after another, its parts.
template <int THREADS, int R, int STEP>
__device__ inline KvShare kv_share(const AttendArgs& a, const KvCrew& crew, int wg, KvShareLds<THREADS>& lds) {
  const int per = (a.n + THREADS - 1) / THREADS, r0 = threadIdx.x * per, r1 = min(a.n, r0 + per);
  long long units = 0;
  int longest = 0;
  KvShare s;
  s.wg = wg;
  s.whole = 0;
  s.mine = 0;
  for (int r = r0; r < r1; ++r) {
    const KvRequest q(a, crew, r);
    if (!q.rows) continue;
    const int n = kv_units<R>(q, a.cache.kv_heads);
    const int steps = kv_unit_steps<STEP>(a, q);
    units += n;
    longest = max(longest, steps);
    s.mine += (long long)n * steps;
  }
  s.all = kv_scan<THREADS>(s.mine, lds.sum, s.before);
  s.per = max((long long)crew.least, kv_quotient(s.all + crew.workgroups - 1, crew.workgroups));
  if (crew.whole) {                          // (the same for all workgroups of the launch)
    long long before;
    const long long n = kv_scan<THREADS>(units, lds.sum, before);
    // Whole units need no join: short ones (two prompts of 1000 to 2000 tokens, 8 heads: 71 us, 132 in shares), and where they fill
    // the machine and none outlasts the others by far.  Else the last ones run alone (three pieces of prompts, 304 units of 66
    // steps: 122 us in shares, 157 whole).
    if (!__syncthreads_or(longest > (n < crew.workgroups ? crew.least : crew.least + 2 * s.per))) {
      s.mine = units;
      s.before = before;
      s.all = n;
      s.whole = s.per = 1;
    }
  }
  s.at = min(s.all, wg * s.per);
  s.end = min(s.all, s.at + s.per);
  return s;
}

// The next part of the share and its request; every thread gets them.
template <int THREADS, int R, int STEP>
__device__ inline KvPart kv_next(const AttendArgs& a, const KvCrew& crew, KvShare& s, KvRequest& q, KvShareLds<THREADS>& lds) {
  KvPart p;
  p.r = -1;
  if (s.at >= s.end) return p;
  const int kv = a.cache.kv_heads;
  __syncthreads();                           // (what was left in LDS for the part before has been read)
  if (s.at >= s.before && s.at < s.before + s.mine) {
    const int per = (a.n + THREADS - 1) / THREADS, r0 = threadIdx.x * per, r1 = min(a.n, r0 + per);
    long long before = s.before;
    for (int r = r0; r < r1; ++r) {
      const KvRequest x(a, crew, r);
      const int steps = kv_unit_steps<STEP>(a, x);
      const long long n = !x.rows ? 0ll : (long long)kv_units<R>(x, kv) * (s.whole ? 1 : steps);
      if (s.at < before + n) {
        lds.r = r;
        lds.first = before;
        lds.unit_steps = steps;
        lds.q = x;
        break;
      }
      before += n;
    }
  }
  __syncthreads();
  p.r = __builtin_amdgcn_readfirstlane(lds.r);
  q.start = __builtin_amdgcn_readfirstlane(lds.q.start);
  q.fresh = __builtin_amdgcn_readfirstlane(lds.q.fresh);
  q.rows = __builtin_amdgcn_readfirstlane(lds.q.rows);
  q.p0 = __builtin_amdgcn_readfirstlane(lds.q.p0);
  q.len = __builtin_amdgcn_readfirstlane(lds.q.len);
  const int tiles = (q.rows + R - 1) / R;
  const long long first = kv_uniform(lds.first), at = s.at - first;
  if (s.whole) {
    // (tiles last to first: a prompt's last rows see the most keys)
    p.tile = tiles - 1 - (int)at / kv;
    p.head = (int)at % kv;
    p.first = 0;
    p.steps = p.count = -1;                  // all, as many as there are
    p.parts = 1;
    s.at = s.end;
    return p;
  }
  p.steps = __builtin_amdgcn_readfirstlane(lds.unit_steps);
  const int unit = (int)kv_quotient(at, p.steps);
  p.head = unit % kv;
  p.tile = unit / kv;
  p.first = (int)(at - (long long)unit * p.steps);
  p.count = (int)min((long long)(p.steps - p.first), s.end - s.at);
  const long long x0 = first + (long long)unit * p.steps;
  p.first_wg = (int)kv_quotient(x0, s.per);
  p.parts = (int)kv_quotient(x0 + p.steps - 1, s.per) - p.first_wg + 1;
  // a unit that goes on is its first workgroup's last part, and any other's first
  p.first_slot = 2 * p.first_wg + (p.first_wg * s.per < x0);
  p.slot = p.first > 0 ? 2 * s.wg : p.first_slot;
  s.at += p.count;
  return p;
}

__device__ inline long long kv_lane(long long v, int lane) {
  return (long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32);
}

// The other way to share: every unit is cut by itself, evenly, into parts of a share's steps at most, one part a workgroup, so
// that units of one part (most, where units are many) meet no other's and leave no partial result.  Every wave finds its
// workgroup's part alone: lane l looks at requests l, l + 64, ...  Requests have one tile (R rows at most).  all: steps of all
// units.  Parts of units that are cut: fewer than 2 all / cut, two shares' number.
template <int STEP>
__device__ inline KvPart kv_cut(const AttendArgs& a, const KvCrew& crew, int wg, KvRequest& q, long long& all) {
  const int lane = threadIdx.x & 63;
  KvRequest own;
  int own_steps = 0;
  const auto look = [&](int r) {
    own = KvRequest(a, crew, r);
    own_steps = own.rows ? kv_unit_steps<STEP>(a, own) : 0;
  };
  const int heads = a.cache.kv_heads;
  all = 0;
  for (int r = lane; r < a.n; r += 64) {
    look(r);
    all += own_steps;
  }
  for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d, 64);
  all = kv_uniform(all) * heads;
  const int cut = (int)min(max((long long)crew.least, kv_quotient(all + crew.workgroups - 1, crew.workgroups)), 1ll << 30);
  // parts, and above them those that leave partial results
  constexpr int SLOTS = 40;
  const auto parts = [&] {
    const long long k = own_steps ? (own_steps - 1) / cut + 1 : 0;
    return heads * (k > 1 ? k | k << SLOTS : k);
  };
  long long mine = 0;
  for (int r = lane; r < a.n; r += 64) {
    if (a.n > 64) look(r);
    mine += parts();
  }
  long long before = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(before, d, 64);
    if (lane >= d) before += o;
  }
  before -= mine;
  constexpr long long LOW = (1ll << SLOTS) - 1;
  const bool here = wg >= (before & LOW) && wg < ((before + mine) & LOW);
  KvPart p;
  p.r = -1;
  const unsigned long long who = __ballot(here);
  if (!who) return p;
  int found = lane;
  if (here)
    for (; found < a.n; found += 64) {
      if (a.n > 64) look(found);
      const long long k = parts();
      if (wg < ((before + k) & LOW)) break;
      before += k;
    }
  const int l = __builtin_ctzll(who);
  p.r = __builtin_amdgcn_readlane(found, l);
  q.start = __builtin_amdgcn_readlane(own.start, l);
  q.fresh = __builtin_amdgcn_readlane(own.fresh, l);
  q.rows = __builtin_amdgcn_readlane(own.rows, l);
  q.p0 = __builtin_amdgcn_readlane(own.p0, l);
  q.len = __builtin_amdgcn_readlane(own.len, l);
  p.steps = __builtin_amdgcn_readlane(own_steps, l);
  before = kv_lane(before, l);
  const int at = wg - (int)(before & LOW);
  p.parts = (p.steps - 1) / cut + 1;
  p.head = at / p.parts;
  const int k = at - p.head * p.parts;
  p.tile = 0;
  p.first = (int)((long long)k * p.steps / p.parts);
  p.count = (int)((long long)(k + 1) * p.steps / p.parts) - p.first;
  p.first_slot = p.first_wg = (int)(before >> SLOTS) + p.head * p.parts;
  p.slot = p.first_slot + k;
  return p;
}

// eight E4M3 codes as a matrix operand of the activation type, exactly
template <int ACT> __device__ inline u32x4_t kv_operand(uint32_t w0, uint32_t w1) {
  u32x4_t o;
  if constexpr (ACT == ACT_F16) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.f, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.f, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.f, true));
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, true));
  }
  return o;
}

// two fp32 values in the activation type, nearest even, in one word
template <int ACT> __device__ inline uint32_t kv_pack(float a, float b) {
  if constexpr (ACT == ACT_F16) {
    half2_t v;
    v[0] = (_Float16)a;
    v[1] = (_Float16)b;
    return __builtin_bit_cast(uint32_t, v);
  } else {
    bf16x2_t v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
  }
}

// sum + the two values of a packed word: the sum of the weights is that of the rounded ones, so that they add up to one
template <int ACT> __device__ inline float kv_add2(uint32_t w, float sum) {
  if constexpr (ACT == ACT_F16) return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, w), half2_t{(_Float16)1.f, (_Float16)1.f}, sum, false);
  else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), bf16x2_t{(__bf16)1.f, (__bf16)1.f}, sum, false);
}

// bytes of w that hold the NaN code: bit 7 of each such byte
__device__ inline uint32_t kv_nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// 1 / l of a finished row.  A row that sees no key is zeros; one whose keys all score -infinity is NaN, as in the formula.
__device__ inline float kv_inverse(float l, const AttendArgs& a, const KvRequest& q, int row) {
  if (l != 0.f) return 1.f / l;
  const int i = row / a.group, lo = a.window ? max(0, q.p0 + i - a.window + 1) : 0;
  return q.hi(i) > lo ? NAN : 0.f;
}

// Eight dims of a finished row, rounded once to the activation type.
template <int ACT, int D>
__device__ inline void kv_store_row(const AttendArgs& a, const KvRequest& q, int head, int row, int d, const float* x) {
  const int i = row / a.group;
  uint16_t* const to = a.out + (size_t)(q.start + i) * a.ldo + ((size_t)head * a.group + (row - i * a.group)) * D + d;
  *(u32x4_t*)to = u32x4_t{kv_pack<ACT>(x[0], x[1]), kv_pack<ACT>(x[2], x[3]), kv_pack<ACT>(x[4], x[5]), kv_pack<ACT>(x[6], x[7])};
}

// partial results go past the XCD's L2
__device__ inline float kv_load_device(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline void kv_store_device(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A unit's rows from their partial results: out = sum w_k o_k / sum w_k, w_k = l_k 2^(M_k - max M).  A result is
// [R][D] o, [R] M, [R] l; the results lie at first_slot, one after another.  A thread takes eight dims of a
// row and, where rows are few, a part of the results; scratch: 10 floats for every thread.
template <int ACT, int D, int R, int THREADS>
__device__ inline void kv_join(const AttendArgs& a, const KvCrew& crew, const KvRequest& q, const KvPart& p, int row0, int rows, float* scratch) {
  constexpr int STRIDE = R * (D + 2);
  const int units = rows * (D / 8);
  int slices = 1;
  while (slices < 16 && 2 * slices * units <= THREADS) slices *= 2;
  for (int u = threadIdx.x; u < units * slices || (slices > 1 && u < THREADS); u += THREADS) {
    const bool live = u < units * slices;
    const int slice = live ? u / units : 0, row = u % units / (D / 8), d = u % (D / 8) * 8;
    float x[8] = {}, top = KV_M_START, sum = 0.f;
    if (live) {
#pragma unroll 4
      for (int k = slice; k < p.parts; k += slices) {
        const float* const from = crew.slots + (size_t)(p.first_slot + k) * STRIDE;
        const float M = kv_load_device(from + R * D + row), l = kv_load_device(from + R * (D + 1) + row);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const unsigned long long v = __hip_atomic_load((const unsigned long long*)(from + row * D + d + e), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          o[e] = __builtin_bit_cast(float, (uint32_t)v);
          o[e + 1] = __builtin_bit_cast(float, (uint32_t)(v >> 32));
        }
        const float most = fmaxf(top, M), f = __builtin_amdgcn_exp2f(top - most), w = l * __builtin_amdgcn_exp2f(M - most);
        top = most;
        sum = __builtin_fmaf(sum, f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(x[e], f, w * o[e]);
      }
    }
    if (slices > 1) {                        // (one round then: all threads are here)
      float* const mine = scratch + threadIdx.x * 10;
#pragma unroll
      for (int e = 0; e < 8; ++e) mine[e] = x[e];
      mine[8] = top;
      mine[9] = sum;
      __syncthreads();
      if (!live || slice > 0) continue;
      for (int k = 1; k < slices; ++k) {
        const float* const other = scratch + (u + k * units) * 10;
        const float most = fmaxf(top, other[8]), f = __builtin_amdgcn_exp2f(top - most), g = __builtin_amdgcn_exp2f(other[8] - most);
        top = most;
        sum = sum * f + other[9] * g;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * f + other[e] * g;
      }
    }
    const float inv = kv_inverse(sum, a, q, row0 + row);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    kv_store_row<ACT, D>(a, q, p.head, row0 + row, d, x);
  }
}

// Four floats of a partial result at device scope (a buffer load, so that the compiler knows of it; 16: past the XCD's L2)
__device__ inline float4_t kv_load4_device(__amdgpu_buffer_rsrc_t slots, uint32_t at) {
  return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(slots, (int)at, 0, 16));
}

// Counts the workgroup in at its unit, once its partial result is out.  Whether it is the unit's last.
__device__ inline bool kv_arrive(const KvCrew& crew, const KvPart& p, uint32_t* arrived) {
  vm_wait<0>();
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t old = __hip_atomic_fetch_add(crew.counts + p.first_wg, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (old == (uint32_t)p.parts - 1) __hip_atomic_store(crew.counts + p.first_wg, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *arrived = old;
  }
  __syncthreads();
  return *arrived == (uint32_t)p.parts - 1;
}

}  // namespace glowq
