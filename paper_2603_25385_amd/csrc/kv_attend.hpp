// Attention over the 8-bit cache: what its kernels share.
//
// Rows.  The `group` q heads of a key/value head and the new tokens of a request are one list of rows, row = token * group
// + head, so that everything that reads a head's keys shares what it has read.  A workgroup takes a tile of rows of one
// (request, key/value head) and a stretch of its keys, a piece.
//
// Pieces.  Lengths are known on the GPU only, so the kernels share out the work themselves: every workgroup adds up the steps
// (stretches of keys) of all requests, takes C = steps / (pieces wanted) as a piece's length, and finds its own piece by its
// index.  What one piece covers whole is stored directly; the pieces of a longer one leave partial results, and the workgroup
// that finds all others of its tile counted joins them in order.
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
  int rows_from, rows_to;        // the kernel serves requests of rows_from < rows <= rows_to
  int pieces, least;             // pieces wanted in all, least steps of one
  uint32_t* counts;              // workspace: arrivals, one word per split tile's first slot
  float* slots;                  // ... partial results
};

// What the kernels know of a request.
struct KvRequest {
  int start, fresh, rows, p0, len;
  __device__ inline KvRequest(const AttendArgs& a, int r) {
    start = min(max(a.starts[r], 0), a.T);
    fresh = min(min(max(a.starts[r + 1] - start, 0), a.max_fresh), a.T - start);
    rows = fresh * a.group;
    if (rows <= a.rows_from || rows > a.rows_to) rows = 0;
    const int length = max(a.lengths[r], 0);
    p0 = length - fresh;
    len = min(length, a.cap);
  }
  // keys [lo, hi) of new tokens i0 .. i1, lo at a 32-token boundary
  __device__ inline int hi(int i1) const { return max(0, min(len, p0 + i1 + 1)); }
  __device__ inline int lo(int i0, int window) const { return window ? max(0, p0 + i0 - window + 1) & ~31 : 0; }
  __device__ inline int steps(int i0, int i1, int window, int step) const {
    const int n = hi(i1) - lo(i0, window);
    return n > 0 ? (n + step - 1) / step : 0;
  }
};

struct KvPiece {
  int r;                 // request; -1: none
  int head, tile;        // key/value head, tile of rows
  int split, splits;     // its place among the tile's pieces
  int per;               // steps of a piece
  int slot;              // of the tile's first partial result; -1: not split
};

template <int THREADS> struct KvPieceShared {
  unsigned long long sum[THREADS / 64];
  KvPiece piece;
};

// sum over the workgroup of v; `before`: over the threads before this one
template <int THREADS>
__device__ inline unsigned long long kv_scan(unsigned long long v, unsigned long long* waves, unsigned long long& before) {
  unsigned long long s = v;
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned long long o = __shfl_up(s, d, 64);
    if ((int)(threadIdx.x & 63) >= d) s += o;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  unsigned long long total = 0;
  before = s - v;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) before += waves[w];
    total += waves[w];
  }
  return total;
}

// The workgroup's piece.  R: rows of a tile, STEP: keys of a step.
template <int THREADS, int R, int STEP>
__device__ inline KvPiece kv_find_piece(const AttendArgs& a, KvPieceShared<THREADS>& sh) {
  const int kv = a.cache.kv_heads;
  const int per_thread = (a.n + THREADS - 1) / THREADS, r0 = threadIdx.x * per_thread, r1 = min(a.n, r0 + per_thread);
  unsigned long long steps = 0, before;
  for (int r = r0; r < r1; ++r) {
    const KvRequest q(a, r);
    if (q.rows) steps += (unsigned long long)((q.rows + R - 1) / R) * q.steps(0, q.fresh - 1, a.window, STEP);
  }
  const unsigned long long all = kv_scan<THREADS>(steps, sh.sum, before) * kv;
  const int per = (int)max((unsigned long long)a.least, (all + a.pieces - 1) / a.pieces);
  // pieces in the low half, slots in the high half
  unsigned long long mine = 0;
  for (int r = r0; r < r1; ++r) {
    const KvRequest q(a, r);
    if (!q.rows) continue;
    const unsigned tiles = kv * ((q.rows + R - 1) / R), splits = max(1, (q.steps(0, q.fresh - 1, a.window, STEP) + per - 1) / per);
    mine += (unsigned long long)(tiles * splits) | (splits > 1 ? (unsigned long long)(tiles * splits) << 32 : 0);
  }
  const unsigned total = (unsigned)kv_scan<THREADS>(mine, sh.sum, before);
  if (threadIdx.x == 0 && blockIdx.x >= total) sh.piece.r = -1;
  unsigned first = (unsigned)before, slot = (unsigned)(before >> 32);
  if (blockIdx.x >= first && blockIdx.x < first + (unsigned)mine)
    for (int r = r0; r < r1; ++r) {
      const KvRequest q(a, r);
      if (!q.rows) continue;
      const unsigned rts = (q.rows + R - 1) / R, splits = max(1, (q.steps(0, q.fresh - 1, a.window, STEP) + per - 1) / per);
      const unsigned n = kv * rts * splits;
      if (blockIdx.x < first + n) {
        const unsigned at = blockIdx.x - first, head = at % kv, rest = at / kv;
        // (tiles last to first: a prompt's last rows see the most keys)
        const unsigned tile = rts - 1 - rest % rts, split = rest / rts;
        sh.piece = KvPiece{r, (int)head, (int)tile, (int)split, (int)splits, per, splits > 1 ? (int)(slot + (tile * kv + head) * splits) : -1};
        break;
      }
      first += n;
      if (splits > 1) slot += n;
    }
  __syncthreads();
  return sh.piece;
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

// Eight dims of a row from its n partial results: out = sum w_k o_k / sum w_k, w_k = l_k 2^(M_k - max M).  o, ml: the first
// one's dims and its M; l lies `l_off` behind M, the next result `stride` behind.
template <int ACT, int D>
__device__ inline void kv_join_row(const AttendArgs& a, const KvRequest& q, int head, int row, int d, const float* o, const float* ml, int l_off,
                                   int stride, int n) {
  float top = KV_M_START;
  for (int k = 0; k < n; ++k) top = fmaxf(top, kv_load_device(ml + (size_t)k * stride));
  float x[8] = {}, sum = 0.f;
#pragma unroll 4
  for (int k = 0; k < n; ++k) {
    const float w = kv_load_device(ml + l_off + (size_t)k * stride) * __builtin_amdgcn_exp2f(kv_load_device(ml + (size_t)k * stride) - top);
    sum += w;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(w, kv_load_device(o + (size_t)k * stride + e), x[e]);
  }
  const float inv = kv_inverse(sum, a, q, row);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= inv;
  kv_store_row<ACT, D>(a, q, head, row, d, x);
}

}  // namespace glowq
