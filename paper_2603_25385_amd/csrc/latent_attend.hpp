// Attention over the latent cache, absorbed: every head's keys and values are the latents themselves.
//
// Rows are (new token, head) pairs of a request, all of which read the same latents; a workgroup takes a tile of 16, 32 or 64 of
// them and a part of the keys (kv_cut, as for the cache of keys and values), 64 keys a step.  A tile of latents lies in LDS once, as
// codes, brought by direct loads two tiles ahead, and serves both products:
//     S^T = K Q^T    a wave's 16 keys, all dims, all rows: q stays in registers, a key's code is read and converted once
//     O^T = C^T P^T  a wave's quarter of the dims, all keys: codes come transposed out of LDS (8 keys of a dim to a lane)
// so that each code is converted twice a tile and no more, whatever the rows.  The weights P go from the first to the second
// through LDS, in 16 bits.
//
// A token's scale 2^e is a factor of its scores' latent part and of its weight: with s = score (base 2), a reference M a row,
//     P = 2^(s - M) 2^e,   O = sum P code,   l = sum 2^(s - M),   out = O / l.
// M follows the largest s + e (with a slack of 2^8, as there), so that the largest weight is about one whatever the scales; l is
// summed up in fp32 from numbers that are at most 2^(8 - e).
//
// A code that is no number makes every score of its token NaN, of rows that do not see it too (before they are masked).  Its row
// of weights then says so to the rows that see it, and the second product takes zeros for such codes: nothing hidden gets through.
#pragma once
#include "kv_attend.hpp"
#include "latent_device.hpp"

namespace glowq {

constexpr int LATENT_STEP = 64, LATENT_STAGES = 3, LATENT_ATTEND_THREADS = 256;

struct LatentAttendArgs {
  AttendArgs a;                // one key/value head, group = heads
  LatentView cache;
};

template <int LATENT, int ROPE, int RG> struct LatentLds {
  uint8_t codes[LATENT_STAGES][LATENT_STEP * LATENT];      // 16-byte chunks of a key's row: chunk c at place c ^ key
  uint8_t ropes[LATENT_STAGES][LATENT_STEP * ROPE * 2];
  uint8_t p[16 * RG * LATENT_STEP * 2];                    // weights [row][key], chunk c of a row at place c ^ row
  float most[4][16 * RG];
  uint32_t odd[LATENT_STAGES];
};

// A partial result: O in the order of the registers, M, l
template <int LATENT, int RG> constexpr int latent_stride() { return 16 * RG * (LATENT + 2); }

__device__ inline u32x4_t lds_read16(const uint8_t* p) { return *(const u32x4_t*)p; }

template <int ACT, int LATENT, int ROPE, int RG>
__device__ inline void latent_part(const LatentAttendArgs& args, const KvCrew& crew, const KvPart& pc, const KvRequest& req, LatentLds<LATENT, ROPE, RG>& lds) {
  constexpr int R = 16 * RG, STEP = LATENT_STEP, CHUNKS = LATENT / 16, ROPE_CHUNKS = ROPE / 8;
  constexpr int CODE_LOADS = 16 * LATENT / 1024, ROPE_LOADS = 16 * ROPE * 2 / 1024, PER = CODE_LOADS + ROPE_LOADS;
  constexpr int LU = LATENT / 64, RU = ROPE / 32, KS = 2 * LU + RU, DG = LATENT / 64;
  const AttendArgs& a = args.a;
  const LatentView& cache = args.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
  const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0);
  const int i0 = scalar(row0 / a.group), i1 = scalar((row0 + rows - 1) / a.group);
  const int begin = pc.first * STEP, end = min(req.hi(i1), begin + pc.count * STEP);
  const int steps = end > begin ? (end - begin + STEP - 1) / STEP : 0;
  const int p_first = req.p0 + i0;

  u32x4_t q[RG][KS];
  int p_row[RG];
#pragma unroll
  for (int b = 0; b < RG; ++b) {
    const int row = min(row0 + 16 * b + c, req.rows - 1), i = row / a.group;
    p_row[b] = req.p0 + i;
    const uint16_t* src = a.q + (size_t)(req.start + i) * a.ldq + (size_t)(row - i * a.group) * (LATENT + ROPE);
#pragma unroll
    for (int u = 0; u < 2 * LU; ++u) q[b][u] = *(const u32x4_t*)(src + 64 * (u >> 1) + 16 * g + 8 * (u & 1));
#pragma unroll
    for (int u = 0; u < RU; ++u) q[b][2 * LU + u] = *(const u32x4_t*)(src + LATENT + 32 * u + 8 * g);
  }

  // Lane n: the block of the wave's 16 keys of step 64 w + n, for the window w at hand and the one behind it; -1: not there
  const auto look_up = [&](int window) {
    const int token = begin + STEP * (64 * window + lane) + 16 * wave;
    const int id = token < end ? a.table[(size_t)pc.r * a.width + (token >> cache.block_shift)] : -1;
    return id < cache.n_blocks ? id : -1;
  };
  int ids = look_up(0), ids_next = look_up(1);
  const auto id_of = [&](int step) { return (step >> 6 & 1) == 0 ? __builtin_amdgcn_readlane(ids, step & 63) : __builtin_amdgcn_readlane(ids_next, step & 63); };
  const auto slot_of = [&](int id, int step) {       // of the first of the wave's keys
    const int token = begin + STEP * step + 16 * wave;
    return id >= 0 ? (size_t)(uint32_t)(id << cache.block_shift) + (token & ((1 << cache.block_shift) - 1)) : (size_t)0;
  };
  const auto bring = [&](int step) {
    const size_t slot = slot_of(id_of(step), step);
    const int stage = step % LATENT_STAGES;
#pragma unroll
    for (int i = 0; i < CODE_LOADS; ++i) {
      constexpr int KEYS = 1024 / LATENT;
      const int key = i * KEYS + lane / CHUNKS, chunk = (lane % CHUNKS) ^ ((16 * wave + key) % CHUNKS);
      lds_dma16(cache.codes + (slot + key) * LATENT + 16 * chunk, lds_address(&lds.codes[stage][(16 * wave + i * KEYS) * LATENT]));
    }
#pragma unroll
    for (int i = 0; i < ROPE_LOADS; ++i) {
      constexpr int KEYS = 512 / ROPE;
      const int key = i * KEYS + lane / ROPE_CHUNKS, chunk = (lane % ROPE_CHUNKS) ^ (key % ROPE_CHUNKS);
      lds_dma16(cache.ropes + (slot + key) * ROPE + 8 * chunk, lds_address(&lds.ropes[stage][(16 * wave + i * KEYS) * ROPE * 2]));
    }
  };
  // scale bytes of keys 4 g .. + 4 of the wave's 16
  const auto look_up_scales = [&](int step) { return *(const uint32_t*)(cache.scales + slot_of(id_of(step), step) + 4 * g); };

  float4_t o[DG][RG];
  float m[RG], l[RG];
#pragma unroll
  for (int b = 0; b < RG; ++b) {
    m[b] = KV_M_START;
    l[b] = 0.f;
#pragma unroll
    for (int d = 0; d < DG; ++d) o[d][b] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (tid < LATENT_STAGES) lds.odd[tid] = 0;
  uint32_t bytes = 0;
  if (steps > 0) {
    bytes = look_up_scales(0);
    bring(0);
    if (steps > 1) bring(1);
  }
  for (int step = 0; step < steps; ++step) {
    const int stage = step % LATENT_STAGES, t0 = begin + STEP * step;
    // this tile has landed, the wave's keys by its own count, the others' by the barrier; and everyone is done with the one before
    if (step + 1 < steps) vm_wait<PER>();
    else vm_wait<0>();
    __syncthreads();
    const int id = id_of(step);
    const uint32_t bytes_now = bytes;
    if (step + 1 < steps) bytes = look_up_scales(step + 1);
    if (step + 2 < steps) bring(step + 2);
    if ((step & 63) == 32) {               // (the window before is done with)
      if ((step >> 6 & 1) == 0) ids_next = look_up((step >> 6) + 1);
      else ids = look_up((step >> 6) + 1);
    }

    // scores of the wave's 16 keys: lane (c, g) has keys 4 g .. + 4 of row c of each block of rows
    float scale[4], exponent[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int byte = id >= 0 ? min(max((int)(bytes_now >> (8 * i) & 255u), 1), 254) : 127;
      scale[i] = kv_pow2(byte - 127);
      exponent[i] = (float)(byte - 127);
    }
    float4_t s[RG];
#pragma unroll
    for (int b = 0; b < RG; ++b) s[b] = float4_t{0.f, 0.f, 0.f, 0.f};
    const uint8_t* const codes = lds.codes[stage] + (16 * wave + c) * LATENT;
#pragma unroll
    for (int u = 0; u < LU; ++u) {
      const u32x4_t w = lds_read16(codes + (((4 * u + g) ^ ((16 * wave + c) % CHUNKS)) * 16));
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const u32x4_t k = kv_operand<ACT>(w[2 * half], w[2 * half + 1]);
#pragma unroll
        for (int b = 0; b < RG; ++b) s[b] = mfma16<ACT>(k, q[b][2 * u + half], s[b]);
      }
    }
#pragma unroll
    for (int b = 0; b < RG; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[b][i] *= scale[i];
    const uint8_t* const ropes = lds.ropes[stage] + (16 * wave + c) * ROPE * 2;
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      const u32x4_t k = lds_read16(ropes + (((4 * u + g) ^ (c % ROPE_CHUNKS)) * 16));
#pragma unroll
      for (int b = 0; b < RG; ++b) s[b] = mfma16<ACT>(k, q[b][2 * LU + u], s[b]);
    }
    const bool all_seen = id >= 0 && t0 + STEP <= end && t0 + STEP - 1 <= p_first;
    float any = 0.f;
#pragma unroll
    for (int b = 0; b < RG; ++b) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        any = __builtin_fmaf(s[b][i], 0.f, any);
        s[b][i] *= a.scale;
        if (!all_seen) {
          const int key = t0 + 16 * wave + 4 * g + i;
          if (id < 0 || key >= end || key > p_row[b]) s[b][i] = -INFINITY;
        }
        top = fmaxf(top, s[b][i] + exponent[i]);
      }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (g == 0) lds.most[wave][16 * b + c] = top;
    }
    if (any != any) lds.odd[stage] = 1;    // (or an infinity: no harm)
    __syncthreads();

    // the weights
#pragma unroll
    for (int b = 0; b < RG; ++b) {
      const int row = 16 * b + c;
      const float top = fmaxf(fmaxf(lds.most[0][row], lds.most[1][row]), fmaxf(lds.most[2][row], lds.most[3][row]));
      if (__any(top > m[b] + KV_M_SLACK)) {
        const float to = fmaxf(top, m[b]), f = __builtin_amdgcn_exp2f(m[b] - to);
        m[b] = to;
        l[b] *= f;
#pragma unroll
        for (int d = 0; d < DG; ++d) o[d][b] *= f;
      }
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(s[b][i] - m[b]);
        l[b] += e;
        p[i] = e * scale[i];
      }
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
      *(u32x2_t*)(lds.p + row * (2 * STEP) + (((2 * wave + (g >> 1)) ^ (c & 7)) * 16) + 8 * (g & 1)) = u32x2_t{kv_pack<ACT>(p[0], p[1]), kv_pack<ACT>(p[2], p[3])};
    }
    const bool odd = lds.odd[stage] != 0;
    __syncthreads();
    if (tid == 0) lds.odd[stage] = 0;      // (read by all; next written two barriers from here)

    // dims 16 (DG wave + d) .. of all rows
    u32x4_t p[2][RG];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int b = 0; b < RG; ++b) p[k][b] = lds_read16(lds.p + (16 * b + c) * (2 * STEP) + (((4 * k + g) ^ (c & 7)) * 16));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int key = 32 * k + 8 * g + (c >> 1);
      const uint8_t* const row = lds.codes[stage] + key * LATENT + 8 * (c & 1);
#pragma unroll
      for (int d = 0; d < DG; ++d) {
        typedef int i32x2_t __attribute__((ext_vector_type(2)));
        const i32x2_t w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2_t*)(row + (((DG * wave + d) ^ (key % CHUNKS)) * 16)));
        uint32_t w0 = (uint32_t)w[0], w1 = (uint32_t)w[1];
        if (__builtin_expect(odd, 0)) {
          w0 &= ~((kv_nan_bytes(w0) >> 7) * 0xffu);
          w1 &= ~((kv_nan_bytes(w1) >> 7) * 0xffu);
        }
        const u32x4_t v = kv_operand<ACT>(w0, w1);
#pragma unroll
        for (int b = 0; b < RG; ++b) o[d][b] = mfma16<ACT>(v, p[k][b], o[d][b]);
      }
    }
  }

  // l of a row: four lanes' keys of four waves
  __syncthreads();
#pragma unroll
  for (int b = 0; b < RG; ++b) {
    l[b] += __shfl_xor(l[b], 16, 64);
    l[b] += __shfl_xor(l[b], 32, 64);
    if (g == 0) lds.most[wave][16 * b + c] = l[b];
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < RG; ++b) {
    const int at = 16 * b + c, row = row0 + at;
    const float sum = (lds.most[0][at] + lds.most[1][at]) + (lds.most[2][at] + lds.most[3][at]);
    if (pc.parts > 1) {
      float* const slot = crew.slots + (size_t)pc.slot * latent_stride<LATENT, RG>();
#pragma unroll
      for (int d = 0; d < DG; ++d) *(float4_t*)(slot + (((wave * DG + d) * RG + b) * 64 + lane) * 4) = o[d][b];
      if (wave == 0 && g == 0) {
        slot[R * LATENT + at] = m[b];
        slot[R * (LATENT + 1) + at] = sum;
      }
    } else if (at < rows) {
      const float inv = kv_inverse(sum, a, req, pc.r, row);
      const int i = row / a.group;
      uint16_t* const to = a.out + (size_t)(req.start + i) * a.ldo + (size_t)(row - i * a.group) * LATENT + 4 * g;
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int d = 0; d < DG; ++d) {
        const float4_t x = o[d][b] * inv;
        *(u32x2_t*)(to + 16 * (DG * wave + d)) = u32x2_t{kv_pack<ACT>(x[0], x[1]), kv_pack<ACT>(x[2], x[3])};
      }
    }
  }
}

}  // namespace glowq
