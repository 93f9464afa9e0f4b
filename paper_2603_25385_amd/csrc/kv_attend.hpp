// Attention over the 8-bit cache: what its kernels share.
//
// Rows.  The `group` q heads of a key/value head and the new tokens of a request are one list of rows, row = token * group
// + head, so that everything that reads a head's keys shares what it has read.  A workgroup takes a tile of rows of one
// (request, key/value head) and a stretch of its keys, a part.
//
// Parts.  Lengths are known on the GPU only, so the kernels share out the work themselves.  A unit is a tile of rows of one
// head of one request, a step a stretch of its keys.  Every unit is cut evenly into parts of a share of all steps at most, and
// the grid has a workgroup for as many parts as there can be.  A unit of one part is stored directly; others leave partial
// results, and the workgroup that finds all others of its unit counted joins them in order.  (Equal shares of all steps in a
// row, which go from unit to unit, cost more than they evened out: 32 requests up to 2000 tokens 29 us, 20 so.)
//
// Scales.  A block's key scale is a factor of its scores; its value scale 2^e is the scale operand of its codes' conversion to the
// matrix cores' type, relative to a reference exponent E that a wave's rows share.  With s = score (base 2) and a reference M
// per row,
//     P = 2^(s - M),   O = sum P (code 2^(e - E)),   l = sum P,   out = O 2^E / l,
// so that what is rounded and summed up as a weight knows nothing of the values.  M is the largest s so far or up to M_SLACK less:
// O and l are rescaled only when a row's s outgrows it by more.  E stays where it is as long as code 2^(e - E) is exact; blocks
// further apart than that have O moved (blocks 2^24 apart at random, binary16: 64 requests up to 8000 tokens 106.5 us, 104.7 without; the
// 8000-token prompt 634, 585 without).
#pragma once
#include "kv_device.hpp"

namespace glowq {

constexpr float KV_M_START = -1.7e38f;    // below every score; finite, so that 2^(-inf - M) is 0
constexpr float KV_M_SLACK = 8.f;         // P <= 2^8: far inside binary16
constexpr float KV_LOG2E = 1.4426950408889634f;
constexpr float KV_L_UNIT = 0x1p-40f;     // of l in a partial result: the sum of results times l stays in fp32, as each does

// Exponents e - E at which every code is a number of the activation type (2^-9 .. 448, NaN), subnormal ones among them; blocks with
// e < ZERO count as zeros: for binary16 their values lie below 2^-32, a hundredth of half its smallest number.
template <int ACT> struct KvRange { static constexpr int HIGH = 7, LOW = ACT == ACT_F16 ? -15 : -117, ZERO = ACT == ACT_F16 ? -40 : KV_EXP_MIN; };
constexpr int KV_KEEP = 64;               // E stays within so much of the largest exponent so far: O stays in fp32
constexpr int KV_ABSENT = -5000, KV_ZEROS = -4999;      // exponents of 16 keys that are not there, of zeros

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
  int shares, least;             // of all steps: how many, and the fewest of one
  int round;                     // workgroups that the machine holds at once, where the shares fill it: as many units as shares are
                                 // cut only where they outlast two of them (0: they are cut all the same)
  uint32_t* counts;              // workspace: arrivals at units that are cut
  float* slots;                  // ... partial results, two per share, of many rows three
  int places;                    // kv_cut with FIT: workgroups that the machine holds at once
};

// What the kernels know of a request.
struct KvRequest {
  int start, fresh, rows, p0, len;
  KvRequest() = default;
  __device__ inline KvRequest(const AttendArgs& a, const KvCrew& crew, int r) {
    // (positions and what is counted back from them stay inside 32 bits, whatever the lengths: keys lie below 2^30)
    const int from = a.starts[r], to = a.starts[r + 1], length = min(max(a.lengths[r], 0), 0x7f000000);
    start = min(max(from, 0), a.T);
    fresh = min(min(max(to - start, 0), a.max_fresh), a.T - start);
    rows = fresh * a.group;
    if (rows <= crew.rows_from || rows > crew.rows_to) rows = 0;
    // (positions go by the tokens that the request brings, those past the bounds among them)
    p0 = max(length - max(to - start, 0), -(1 << 30));
    len = min(length, a.cap);
  }
  // keys [lo, hi) of new tokens i0 .. i1, lo at a 32-token boundary
  __device__ inline int hi(int i1) const { return max(0, min(len, p0 + i1 + 1)); }
  __device__ inline int lo(int i0, int window) const { return window ? max(0, min(p0 + i0 - window + 1, len)) & ~31 : 0; }
  // ... in steps, one at least
  __device__ inline int steps(int i0, int i1, int window, int step) const {
    const int n = hi(i1) - lo(i0, window);
    return n > 0 ? (n + step - 1) / step : 1;
  }
};

// A workgroup's part of a unit: steps first .. first + count.  parts: of the unit; their partial results lie at first_slot, one
// after another (this one's at slot), and are counted at that word.
struct KvPart {
  int r, head, tile;             // r < 0: none
  int first, count;
  int parts, first_slot, slot;
  int slots;                     // partial results of all units; set where r is not
};

// v / by, both positive (the division of 64 bits takes five times as long)
__device__ inline long long kv_quotient(long long v, long long by) {
  return (v | by) >> 32 ? v / by : (long long)((uint32_t)v / (uint32_t)by);
}

// Units of a request, and the steps that each is taken to have (those of its last rows: the most)
template <int R> __device__ inline int kv_units(const KvRequest& q, int kv_heads) { return (q.rows + R - 1) / R * kv_heads; }
template <int STEP> __device__ inline int kv_unit_steps(const AttendArgs& a, const KvRequest& q) { return q.steps(0, q.fresh - 1, a.window, STEP); }

__device__ inline long long kv_lane(long long v, int lane) {
  return (long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32);
}

// Sums over lanes 0 .. l, in lane l (rows of 16 by themselves, then rows joined; moved across lanes by the vector ALU: by way of LDS, as shuffles
// go, single tokens took 0.3 to 0.7 us longer)
template <int CTRL, int ROWS> __device__ inline long long kv_scan_step(long long v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, true);
  return v + (long long)((uint64_t)hi << 32 | lo);
}
__device__ inline long long kv_scan(long long v) {
  v = kv_scan_step<0x111, 0xf>(v);         // lanes 1, 2, 4, 8 below in the row
  v = kv_scan_step<0x112, 0xf>(v);
  v = kv_scan_step<0x114, 0xf>(v);
  v = kv_scan_step<0x118, 0xf>(v);
  v = kv_scan_step<0x142, 0xa>(v);         // the last of the row before, for rows 1 and 3
  return kv_scan_step<0x143, 0xc>(v);      // lane 31, for rows 2 and 3
}

// The workgroup's part.  Every unit is cut by itself, evenly, into parts of a share's steps at most, one part a workgroup, so that
// units of one part (most, where units are many) leave no partial result and no workgroup goes from unit to unit.  Every wave
// finds the part alone: lane l looks at requests l, l + 64, ...  all: steps of all units, as they are taken; total: parts.
// Parts of cut units are fewer than 2 all / cut, two for every share.  Parts that would fill a second round of the machine by less
// than half are made smaller by a third, which at most doubles them: three for every share.  Over 44 batches, 41 of them drawn at random, that is
// 0.4 % less time in the mean: 203 -> 170 us (3 x 160 tokens on 20000, 32 heads), 206 -> 176 (712 on 13000), 139 -> 128 (3 x 500 on 16000 in
// windows of 4096), but 97 -> 108 (365 on 8000 beside 4 decoding, 32 heads) and 74 -> 79 (3 x 196 on 3900, 40 heads).  Heads of 64, of which
// the machine holds 768 workgroups, would lose by the 512 of heads of 128: 40 us, 49 so (40 decoding sequences beside a prompt of 1500).
// FIT (kernels of few, large workgroups): parts are made larger, from an equal share of all steps on, until they fit into whole rounds of the
// machine, by an eighth each time (nearer costs as much as it gives); one round where units are fewer than three quarters of its
// places, and so on.  (One round up to all of its places: 112 requests of up to 4000 tokens, 128 heads 157 us for 141, 210 of up to 6000, 64 heads 217 for 183,
// but 124 of up to 2000, 128 heads 93 for 97.)
template <int R, int STEP, bool FIT = false>
__device__ inline KvPart kv_cut(const AttendArgs& a, const KvCrew& crew, int wg, KvRequest& q, long long& all, long long& total) {
  const int lane = threadIdx.x & 63;
  KvRequest own;
  int own_steps = 0;
  const auto look = [&](int r) {
    own = KvRequest(a, crew, r);
    own_steps = own.rows ? kv_unit_steps<STEP>(a, own) : 0;
  };
  const int heads = a.cache.kv_heads;
  long long units = 0;
  all = 0;
  for (int r = lane; r < a.n; r += 64) {
    look(r);
    units += kv_units<R>(own, heads);
    all += (long long)kv_units<R>(own, heads) * own_steps;
  }
  all = kv_lane(kv_scan(all), 63);
  units = kv_lane(kv_scan(units), 63);
  long long share = max((long long)crew.least, kv_quotient(all + crew.shares - 1, crew.shares));
  if (crew.round && units >= crew.shares) share = 2 * share + crew.least;
  // parts, and above them those that leave partial results
  long long room = 0;
  if constexpr (FIT) {
    room = crew.places * (1 + kv_quotient(4 * units + crew.places, 4 * crew.places));
    share = max((long long)crew.least, kv_quotient(all + room - 1, room));
  }
  constexpr int SLOTS = 40;
  constexpr long long LOW = (1ll << SLOTS) - 1;
  int cut = (int)min(share, 1ll << 30);
  const auto parts = [&] {
    const long long k = own_steps ? (own_steps - 1) / cut + 1 : 0;
    return kv_units<R>(own, heads) * (k > 1 ? k | k << SLOTS : k);
  };
  long long mine, before, sums;
  for (;;) {
    mine = 0;
    for (int r = lane; r < a.n; r += 64) {
      if (a.n > 64) look(r);
      mine += parts();
    }
    before = kv_scan(mine);
    sums = kv_lane(before, 63);
    total = sums & LOW;
    if constexpr (FIT) {
      if (total <= room || cut >= 1 << 29) break;
      cut += (cut >> 3) + 1;
      continue;
    }
    if (!crew.round || total <= crew.round || 2 * total >= 3 * crew.shares || cut < 2 * crew.least || cut < share) break;
    cut = cut * 2 / 3;
  }
  before -= mine;
  const bool here = wg >= (before & LOW) && wg < ((before + mine) & LOW);
  KvPart p;
  p.r = -1;
  p.slots = (int)(sums >> SLOTS);
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
  before = kv_lane(before, l);
  // (quotients come from the vector ALU: back to scalar registers)
  const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int at = scalar(wg - (int)(before & LOW));
  p.parts = scalar((__builtin_amdgcn_readlane(own_steps, l) - 1) / cut + 1);
  const int unit = scalar(at / p.parts), k = at - unit * p.parts, turn = scalar(unit / heads);
  // (tiles last to first: a prompt's last rows see the most keys)
  p.tile = (q.rows - 1) / R - turn;
  p.head = unit - turn * heads;
  const int i0 = scalar(p.tile * R / a.group), i1 = scalar((min(q.rows, p.tile * R + R) - 1) / a.group);
  const int steps = q.steps(i0, i1, a.window, STEP);
  p.first = scalar((int)(kv_quotient((long long)k * steps, p.parts)));
  p.count = scalar((int)(kv_quotient((long long)(k + 1) * steps, p.parts))) - p.first;
  p.first_slot = scalar((int)(before >> SLOTS)) + unit * p.parts;
  p.slot = p.first_slot + k;
  return p;
}

// eight E4M3 codes as a matrix operand of the activation type, four times s0 and four times s1 (powers of two)
template <int ACT> __device__ inline u32x4_t kv_operand(uint32_t w0, uint32_t w1, float s0 = 1.f, float s1 = 1.f) {
  u32x4_t o;
  if constexpr (ACT == ACT_F16) {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, s0, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, s0, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, s1, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, s1, true));
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s0, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s0, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s1, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s1, true));
  }
  return o;
}

// The reference exponent of a wave's sums O, and the largest exponent that it has been moved for
struct KvReference { int at, top; };

// Whether values of exponent e need more than a scale of 2^(e - E): they are not exact so, or they are zeros or not there
template <int ACT> __device__ inline bool kv_wild(int e, int at) {
  using Range = KvRange<ACT>;
  return (uint32_t)(e - at - Range::LOW) > (uint32_t)(Range::HIGH - Range::LOW);
}
// That scale
__device__ inline float kv_value_scale(int e, int at) { return kv_pow2(min(max(e - at, -126), 126)); }

// Moves the reference to exponent e, or near it.  move(d): O times 2^d.
template <class Move> __device__ inline void kv_refer(int e, KvReference& ref, Move move) {
  ref.top = max(ref.top, e);
  const int to = max(e, ref.top - KV_KEEP);
  if (to != ref.at) move(ref.at - to);
  ref.at = to;
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

// 1 / l of a finished row.  A row that sees no key, or whose keys all lie in blocks outside the cache, is zeros; one whose keys all
// score -infinity is NaN, as in the formula.
__device__ inline float kv_inverse(float l, const AttendArgs& a, const KvRequest& q, int r, int row) {
  if (l != 0.f) return 1.f / l;
  const int i = row / a.group, lo = a.window ? max(0, q.p0 + i - a.window + 1) : 0, hi = q.hi(i);
  for (int b = lo >> a.cache.block_shift; lo < hi && b <= (hi - 1) >> a.cache.block_shift; ++b)
    if ((uint32_t)a.table[(size_t)r * a.width + b] < (uint32_t)a.cache.n_blocks) return NAN;
  return 0.f;
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
    const float inv = kv_inverse(sum, a, q, p.r, row0 + row);
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
    const uint32_t old = __hip_atomic_fetch_add(crew.counts + p.first_slot, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (old == (uint32_t)p.parts - 1) __hip_atomic_store(crew.counts + p.first_slot, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *arrived = old;
  }
  __syncthreads();
  return *arrived == (uint32_t)p.parts - 1;
}

}  // namespace glowq
