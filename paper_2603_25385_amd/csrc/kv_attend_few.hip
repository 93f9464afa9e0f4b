// Attention over the 8-bit cache for few rows per (request, key/value head): single tokens, short pieces of a prompt.
#include <algorithm>
#include "kv_attend.hpp"
#include "kv_attend_host.hpp"

namespace glowq {

constexpr int FEW_THREADS = 256, FEW_WAVES = FEW_THREADS / 64;
constexpr int FEW_KEYS = 32;                          // of a wave's tile
constexpr int FEW_STEP = FEW_KEYS * FEW_WAVES;

// Keys and values of 32 tokens as they lie in the cache: [16-token tile][64 dims]
template <int DP> struct KvTile {
  u32x4_t k[2][DP], v[2][DP];
};

template <int ACT, int DP, int RB>
__global__ void __launch_bounds__(FEW_THREADS) k_kv_attend_few(AttendArgs a) {
  constexpr int R = 16 * RB, D = 64 * DP, LD = D + 4;             // (rows of LDS 16 bytes apart in their banks)
  __shared__ KvPieceShared<FEW_THREADS> piece_lds;
  __shared__ float o_lds[2][R][LD];
  __shared__ float m_lds[FEW_WAVES][R], l_lds[FEW_WAVES][R];
  __shared__ uint32_t arrived;
  const KvPiece pc = kv_find_piece<FEW_THREADS, R, FEW_STEP>(a, piece_lds);
  if (pc.r < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, g = lane >> 4;
  const KvRequest req(a, pc.r);
  const KvView& cache = a.cache;
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0);
  const int i0 = row0 / a.group, i1 = (row0 + rows - 1) / a.group;
  const int steps = req.steps(i0, i1, a.window, FEW_STEP);
  const int n_pieces = max(1, (steps + pc.per - 1) / pc.per);
  if (pc.split >= n_pieces) return;
  const int begin = req.lo(i0, a.window) + pc.split * pc.per * FEW_STEP;
  const int end = min(req.hi(i1), begin + pc.per * FEW_STEP);
  const int p_first = req.p0 + i0, p_last = req.p0 + i1;

  u32x4_t q[RB][DP][2];
  int p_row[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int row = row0 + 16 * b + c16, i = row / a.group;
    p_row[b] = req.p0 + i;
    const bool live = row < req.rows;
    const uint16_t* src = a.q + (size_t)(req.start + (live ? i : i0)) * a.ldq + ((size_t)pc.head * a.group + (live ? row - i * a.group : 0)) * D + 16 * g;
#pragma unroll
    for (int d = 0; d < DP; ++d)
#pragma unroll
      for (int h = 0; h < 2; ++h) q[b][d][h] = *(const u32x4_t*)(src + 64 * d + 8 * h);
  }
  float4_t o[RB][DP * 4];
  float m[RB], l[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    m[b] = KV_M_START;
    l[b] = 0.f;
#pragma unroll
    for (int d = 0; d < DP * 4; ++d) o[b][d] = float4_t{0.f, 0.f, 0.f, 0.f};
  }

  const int tiles = end > begin ? (end - begin + FEW_KEYS - 1) / FEW_KEYS : 0;      // of all waves
  const int mine = tiles > wave ? (tiles - wave + FEW_WAVES - 1) / FEW_WAVES : 0;
  for (int k0 = 0; k0 < mine; k0 += 32) {
    // lane 2 k + s: where 16-token tile s of this wave's tile k0 + k lies, and its scales
    const int token = begin + (wave + FEW_WAVES * (k0 + (lane >> 1))) * FEW_KEYS + 16 * (lane & 1);
    int id = token < end ? a.table[(size_t)pc.r * a.width + (token >> cache.block_shift)] : -1;
    const bool ok = id >= 0 && id < cache.n_blocks;
    if (!ok) id = 0;
    const size_t at = cache.page(id, pc.head) + (ok ? (size_t)((token & ((1 << cache.block_shift) - 1)) >> 4) * DP * KV_PIECE : 0);
    const uint32_t at_lo = (uint32_t)at, at_hi = (uint32_t)(at >> 32);
    const size_t sc = (size_t)id * cache.kv_heads + pc.head;
    const uint32_t info = (uint32_t)cache.scales[0][sc] | (uint32_t)cache.scales[1][sc] << 8 | (ok ? 1u << 16 : 0u);

    const auto fetch = [&](int k, KvTile<DP>& t) {
      k = min(k, 31);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const size_t off = (size_t)(uint32_t)__builtin_amdgcn_readlane(at_lo, 2 * k + s) | (size_t)(uint32_t)__builtin_amdgcn_readlane(at_hi, 2 * k + s) << 32;
        const u32x4_t* kp = (const u32x4_t*)(cache.codes[0] + off);
        const u32x4_t* vp = (const u32x4_t*)(cache.codes[1] + off);
#pragma unroll
        for (int d = 0; d < DP; ++d) {
          t.k[s][d] = kp[64 * d + lane];
          t.v[s][d] = vp[64 * d + lane];
        }
      }
    };
    const auto run = [&](int k, KvTile<DP>& t) {
      const int t0 = begin + (wave + FEW_WAVES * (k0 + k)) * FEW_KEYS;
      const uint32_t in[2] = {(uint32_t)__builtin_amdgcn_readlane(info, 2 * k), (uint32_t)__builtin_amdgcn_readlane(info, 2 * k + 1)};
      float4_t s[RB][2];
#pragma unroll
      for (int b = 0; b < RB; ++b) s[b][0] = s[b][1] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int d = 0; d < DP; ++d)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const u32x4_t x = kv_operand<ACT>(t.k[h][d][2 * u], t.k[h][d][2 * u + 1]);
#pragma unroll
            for (int b = 0; b < RB; ++b) s[b][h] = mfma16<ACT>(x, q[b][d][u], s[b][h]);
          }
      const bool whole = (in[0] & in[1] & 1u << 16) && t0 + FEW_KEYS - 1 <= p_first && t0 + FEW_KEYS <= end && (!a.window || t0 > p_last - a.window);
      uint32_t nan_bytes = 0;
      if (!whole) {
        // hidden keys: no score, no value; what lies behind the last token may be anything
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = t0 + 16 * h + 4 * g;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int b = 0; b < RB; ++b) {
              const bool seen = (in[h] & 1u << 16) && key + e < end && key + e <= p_row[b] && (!a.window || key + e > p_row[b] - a.window);
              s[b][h][e] = seen ? s[b][h][e] : -INFINITY;
            }
          const int left = (in[h] & 1u << 16) ? min(4, max(0, end - key)) : 0;       // of the lane's four tokens
          const uint32_t keep = left > 0 ? 0xffffffffu >> (8 * (4 - left)) : 0u;
#pragma unroll
          for (int d = 0; d < DP; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              t.v[h][d][j] &= keep;
              nan_bytes |= kv_nan_bytes(t.v[h][d][j]);
            }
        }
      }
      const float ka[2] = {kv_pow2((int)(in[0] & 255u) - 127) * a.scale, kv_pow2((int)(in[1] & 255u) - 127) * a.scale};
      const float ve[2] = {(float)((int)(in[0] >> 8 & 255u) - 127), (float)((int)(in[1] >> 8 & 255u) - 127)};
      const float vi[2] = {kv_pow2(127 - (int)(in[0] >> 8 & 255u)), kv_pow2(127 - (int)(in[1] >> 8 & 255u))};
      u32x4_t p[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        float top[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          top[h] = fmaxf(fmaxf(s[b][h][0], s[b][h][1]), fmaxf(s[b][h][2], s[b][h][3])) * ka[h] + ve[h];
        float most = fmaxf(top[0], top[1]);
        if (__any(most > m[b] + KV_M_SLACK)) {
          most = fmaxf(most, __shfl_xor(most, 16, 64));
          most = fmaxf(most, __shfl_xor(most, 32, 64));
          most = fmaxf(most, m[b]);
          const float f = __builtin_amdgcn_exp2f(m[b] - most);
          m[b] = most;
          l[b] *= f;
#pragma unroll
          for (int d = 0; d < DP * 4; ++d) o[b][d] *= f;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][h][i], ka[h], ve[h] - m[b]));
          l[b] = __builtin_fmaf((e[0] + e[1]) + (e[2] + e[3]), vi[h], l[b]);
          p[b][2 * h] = kv_pack<ACT>(e[0], e[1]);
          p[b][2 * h + 1] = kv_pack<ACT>(e[2], e[3]);
        }
      }
      const bool odd = !whole && __any(nan_bytes != 0);
      if (odd) {
        // a value that is not a number, seen by some rows only: 0 * NaN must not reach the others.  The rows that see it are
        // those where (seen) * (is NaN) sums to more than nothing
        constexpr uint32_t ONE = ACT == ACT_F16 ? 0x3c00u : 0x3f80u;
#pragma unroll
        for (int d = 0; d < DP; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            u32x4_t is;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t n = kv_nan_bytes(t.v[h][d][j]);
              is[2 * h] = (n & 0x80u ? ONE : 0u) | (n & 0x8000u ? ONE << 16 : 0u);
              is[2 * h + 1] = (n & 0x800000u ? ONE : 0u) | (n & 0x80000000u ? ONE << 16 : 0u);
              t.v[h][d][j] &= ~((n >> 7) * 0xffu);
            }
#pragma unroll
            for (int b = 0; b < RB; ++b) {
              u32x4_t seen;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float lo = s[b][i >> 1][(i & 1) * 2], hi = s[b][i >> 1][(i & 1) * 2 + 1];
                seen[i] = (lo != -INFINITY ? ONE : 0u) | (hi != -INFINITY ? ONE << 16 : 0u);
              }
              const float4_t hit = mfma16<ACT>(is, seen, float4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (hit[i] > 0.f) o[b][4 * d + j][i] = NAN;
            }
          }
      }
#pragma unroll
      for (int d = 0; d < DP; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4_t x = kv_operand<ACT>(t.v[0][d][j], t.v[1][d][j]);
#pragma unroll
          for (int b = 0; b < RB; ++b) o[b][4 * d + j] = mfma16<ACT>(x, p[b], o[b][4 * d + j]);
        }
    };
    const int here = min(32, mine - k0);
    KvTile<DP> t[2];
    fetch(0, t[0]);
    fetch(1, t[1]);
    for (int k = 0; k < here; k += 2) {
      run(k, t[0]);
      fetch(k + 2, t[0]);
      if (k + 1 < here) run(k + 1, t[1]);
      fetch(k + 3, t[1]);
    }
  }

  // the waves' results become one: the rows' largest reference, then sums of two waves each through LDS
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    l[b] += __shfl_xor(l[b], 16, 64);
    l[b] += __shfl_xor(l[b], 32, 64);
    if (g == 0) {
      m_lds[wave][16 * b + c16] = m[b];
      l_lds[wave][16 * b + c16] = l[b];
    }
  }
  __syncthreads();
  float f[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int row = 16 * b + c16;
    const float top = fmaxf(fmaxf(m_lds[0][row], m_lds[1][row]), fmaxf(m_lds[2][row], m_lds[3][row]));
    f[b] = __builtin_amdgcn_exp2f(m[b] - top);
  }
#pragma unroll
  for (int turn = 0; turn < 2; ++turn) {
    if ((wave >> 1) == 1 - turn)
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int d = 0; d < DP * 4; ++d) {
          float4_t* to = (float4_t*)&o_lds[wave & 1][16 * b + c16][16 * d + 4 * g];
          const float4_t x = o[b][d] * f[b];
          *to = turn ? x + *to : x;
        }
    __syncthreads();
  }
  // rows out, or a partial result: eight dims a thread
  const bool split = n_pieces > 1;
  float* const slot = split ? a.slots + (size_t)(pc.slot + pc.split) * (R * (D + 2)) : nullptr;
  for (int u = tid; u < rows * (D / 8); u += FEW_THREADS) {
    const int row = u / (D / 8), d = u % (D / 8) * 8;
    const float top = fmaxf(fmaxf(m_lds[0][row], m_lds[1][row]), fmaxf(m_lds[2][row], m_lds[3][row]));
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) sum += l_lds[w][row] * __builtin_amdgcn_exp2f(m_lds[w][row] - top);
    float x[8];
    const float inv = !split ? kv_inverse(sum, a, req, row0 + row) : sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (o_lds[0][row][d + e] + o_lds[1][row][d + e]) * inv;
    if (!split) kv_store_row<ACT, D>(a, req, pc.head, row0 + row, d, x);
    else {
#pragma unroll
      for (int e = 0; e < 8; e += 4) store16_device(slot + row * D + d + e, __builtin_bit_cast(u32x4_t, float4_t{x[e], x[e + 1], x[e + 2], x[e + 3]}));
      if (d == 0) {
        kv_store_device(slot + R * D + row, top);
        kv_store_device(slot + R * (D + 1) + row, sum);
      }
    }
  }
  if (!split) return;
  vm_wait<0>();
  __syncthreads();
  if (tid == 0) arrived = __hip_atomic_fetch_add(a.counts + pc.slot, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (arrived != (uint32_t)n_pieces - 1) return;
  if (tid == 0) __hip_atomic_store(a.counts + pc.slot, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const float* const first = a.slots + (size_t)pc.slot * (R * (D + 2));
  for (int u = tid; u < rows * (D / 8); u += FEW_THREADS) {
    const int row = u / (D / 8), d = u % (D / 8) * 8;
    kv_join_row<ACT, D>(a, req, pc.head, row0 + row, d, first + row * D + d, first + R * D + row, R, R * (D + 2), n_pieces);
  }
}

template <int ACT, int DP, int RB> static void go(const AttendArgs& a, int grid, hipStream_t st) {
  k_kv_attend_few<ACT, DP, RB><<<dim3(grid), dim3(FEW_THREADS), 0, st>>>(a);
}
hipError_t launch_kv_attend_few(const AttendArgs& a, int act, int blocks_of_rows, int grid, hipStream_t st) {
  const int dp = 1 << (a.cache.dim_shift - 6);
#define GLOWQ_FEW(DP, RB) \
  if (dp == DP && blocks_of_rows == RB) act == GLOWQ_F16 ? go<ACT_F16, DP, RB>(a, grid, st) : go<ACT_BF16, DP, RB>(a, grid, st)
  GLOWQ_FEW(1, 1);
  GLOWQ_FEW(2, 1);
  GLOWQ_FEW(1, 2);
  GLOWQ_FEW(2, 2);
#undef GLOWQ_FEW
  return hipGetLastError();
}

}  // namespace glowq
