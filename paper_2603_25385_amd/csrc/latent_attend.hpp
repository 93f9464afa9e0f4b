// Attention over the latent cache, absorbed: every head's keys and values are the latents themselves.
//
// Rows are (new token, head) pairs of a request, all of which read the same latents; a workgroup takes a tile of 16, 32 or 64 of
// them and a part of the keys (kv_cut, as for the cache of keys and values), 64 keys a step.  A tile of latents lies in LDS once, as
// codes, brought by direct loads one to two tiles ahead, and serves both products:
//     S^T = K Q^T    a wave has 16 keys, all dims, and all rows or half of them: q stays in registers, a code is read for both halves
//     O^T = C^T P^T  a wave has an equal share of the dims, all keys and rows: codes come transposed out of LDS (8 keys of a dim to a lane)
// so that a code is converted two or three times a tile, whatever the rows.  The weights P go from the first to the second
// through LDS, in 16 bits.  16 rows take four waves; more take eight, two to a SIMD, so that all that a wave keeps fits into 256
// registers (four waves with 512: sums moved to accumulation registers and back, 346 us for 64 requests of up to 8000 tokens, 128 heads).
//
// A token's scale 2^e is a factor of its scores' latent part and of its weight: with s = score (base 2), a reference M a row,
//     w = 2^(s - M) rounded to the type's bits,   P = w 2^e,   O = sum P code,   l = sum w,   out = O / l.
// M stays until a row's largest s + e has outgrown it by 2^8 (as there), so that the largest P is near one whatever the scales; in binary16
// it is 2^7 to 2^15, the upper end of the type, so that weights keep all bits down to 2^-21 of the largest and some down to 2^-31.  (100000 tokens
// behind one that weighs 2^22, 2^24 or 2^26 of theirs and adds nothing to O: error 2.6e-4, 2.5e-4, 3.3e-4 of the output.  With the largest at 2^0 to
// 2^8 it was 3.9e-3, 2e-2, 1: what O had lost was still in l.)  l's
// numbers are then about 2^-e, e from -64 to 120: it is summed up 2^24 times as large, in the middle of fp32's range.
//
// A code that is no number makes every score of its token NaN, of rows that do not see it too (before they are masked).  Its row
// of weights then says so to the rows that see it, and the second product takes zeros for such codes (of a tile that has something to
// hide): nothing hidden gets through.
//
// Bound.  64 requests of up to 8000 tokens, 128 heads, latents of 512, bfloat16: 130 us, 0.61 PFLOP/s, 2.6 us for 64 rows and 64 keys: vector ALU,
// products and LDS one behind another in every wave, the first the most; what took instructions from a tile took time (144 us with
// references looked at for every score and scores scaled by themselves).  No faster: weights made between two barriers, by references that
// the waves found together (152 when this took 144); half of the waves with scores first, half with the second product first (153); codes
// as they are on the 8-bit instructions with q and the weights in two parts (no conversions, 160 to 179); 32 rows, half of the keys
// and all dims to a wave (latents of 256 the same; of 512 one wave issues too many instructions, 208); six tiles in LDS
// for latents of 256 (the same).
#pragma once
#include "kv_attend.hpp"
#include "latent_device.hpp"
#include "wide.hpp"

namespace glowq {

constexpr int LATENT_STEP = 64, LATENT_STAGES = 3;
constexpr float LATENT_LIFT = 24.f, LATENT_LIFTED = 0x1p24f;         // of l in the kernel and in partial results
// The largest P of a row is 2^BITS where its reference is new.  One above 2^8 of that (and what rounding adds) says that its row needs a new reference.  Rows
// get one from 2^8.06 on: any such row says so by itself, so that no other row changes its bits.
template <int ACT> struct LatentHeld {
  static constexpr float BITS = ACT == ACT_F16 ? 7.f : 0.f, GROWN = ACT == ACT_F16 ? 0x1.06p15f : 0x1.06p8f;
};
constexpr int latent_waves(int RG) { return RG == 1 ? 4 : 8; }

// Stretches of 32 dims at the queries' end, the rope part's among them, that lie in LDS: where registers do not hold all
constexpr int latent_queries_in_lds(int LATENT, int ROPE, int RG) { return LATENT == 512 && RG == 4 ? (ROPE / 32 + 3) / 2 * 2 : 0; }

struct LatentAttendArgs {
  AttendArgs a;                // one key/value head, group = heads
  LatentView cache;
};

// (what is read at fixed places comes first: its offsets fit into the instructions)
template <int LATENT, int ROPE, int RG> struct alignas(16) LatentLds {
  uint8_t p[2][16 * RG * LATENT_STEP * 2];                 // weights [row][key] of two tiles, chunk c of a row at place c ^ row
  float4_t most[16 * RG];                                  // of a row's keys, 16 each
  uint32_t scales[LATENT_STAGES][LATENT_STEP / 4];
  uint32_t odd[4], grown[4];                               // of a stage: codes that may be no numbers; a row that needs a new reference
  uint8_t q[latent_queries_in_lds(LATENT, ROPE, RG) * 16 * RG * 64 + 16];          // 32 dims of a row; chunk c at place c ^ row / 2
  struct {
    uint8_t codes[LATENT_STEP * LATENT];                   // 16-byte chunks of a key's row: chunk c at place c ^ key
    uint8_t ropes[LATENT_STEP * ROPE * 2];
  } stage[LATENT_STAGES];
};

// A partial result: O in the order of the registers, M, l
template <int LATENT, int RG> constexpr int latent_stride() { return 16 * RG * (LATENT + 2); }

// a value that the compiler must take as new: what is made of it is not kept over a loop's rounds (where registers are short)
template <bool SHORT = true> __device__ inline int made_anew(int v) {
  if constexpr (SHORT) asm volatile("" : "+v"(v));
  return v;
}

// A number of any size to as many significant bits as binary16 has (halfway cases away from zero; what a 16-bit NaN becomes stays NaN)
__device__ inline float latent_round11(float v) { return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, v) + 0x1000u) & 0xffffe000u); }

// the largest of lanes c, c + 16, c + 32, c + 48
__device__ inline float max_of_groups(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

__device__ inline u32x4_t lds_read16(const uint8_t* p) { return *(const u32x4_t*)p; }

// The keys of a part, as a wave sees them: 16 of every tile.  Blocks are looked up 64 steps ahead, a lane a step.
template <int LATENT, int ROPE, int RG> struct LatentKeys {
  static constexpr int WAVES = latent_waves(RG), HALVES = WAVES / 4, STEP = LATENT_STEP, CHUNKS = LATENT / 16, ROPE_CHUNKS = ROPE / 8;
  static constexpr bool SHORT = LATENT == 512 && RG == 4;          // of registers
  // what a wave brings of a tile: all codes of its keys, or a half where another wave has the same keys; their key parts (32 numbers
  // are one load for 16 keys: both waves bring the same); their scales
  static constexpr int KEYS = 16 / HALVES, CODE_LOADS = KEYS * LATENT / 1024, ROPE_LOADS = HALVES == 2 || ROPE == 32 ? 1 : 2, PER = CODE_LOADS + ROPE_LOADS + 1;
  LatentLds<LATENT, ROPE, RG>& lds;
  const uint8_t *codes, *all_scales;
  const uint16_t* ropes;
  const int32_t* blocks;       // the request's row of the table
  int n_blocks, block_shift, begin, end, kg, half, lane;
  int ids, ids_next;           // of step 64 w + lane, of the window w at hand and of the one behind it; -1: not there

  __device__ __attribute__((always_inline)) inline LatentKeys(LatentLds<LATENT, ROPE, RG>& to, const LatentAttendArgs& x, const KvPart& pc, int from, int until)
      : lds(to), codes(x.cache.codes), all_scales(x.cache.scales), ropes(x.cache.ropes), blocks(x.a.table + (size_t)pc.r * x.a.width), n_blocks(x.cache.n_blocks),
        block_shift(x.cache.block_shift), begin(from), end(until) {
    lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    kg = wave & 3;
    half = wave >> 2;
    ids = look_up(0);
    ids_next = look_up(1);
  }
  __device__ __attribute__((always_inline)) inline int look_up(int window) const {
    const int token = begin + STEP * (64 * window + lane) + 16 * kg;
    const int id = token < end ? blocks[token >> block_shift] : -1;
    return id < n_blocks ? id : -1;
  }
  __device__ __attribute__((always_inline)) inline void look_ahead(int step) {
    if ((step & 63) != 32) return;         // (the window before is done with)
    if ((step >> 6 & 1) == 0) ids_next = look_up((step >> 6) + 1);
    else ids = look_up((step >> 6) + 1);
  }
  __device__ __attribute__((always_inline)) inline int id_of(int step) const {
    return __builtin_amdgcn_readlane((step >> 6 & 1) == 0 ? ids : ids_next, step & 63);
  }
  __device__ __attribute__((always_inline)) inline size_t slot_of(int step) const {       // of the first of the wave's keys
    const int token = begin + STEP * step + 16 * kg, id = id_of(step);
    return id >= 0 ? (size_t)(uint32_t)(id << block_shift) + (token & ((1 << block_shift) - 1)) : (size_t)0;
  }
  // load i of PER
  __device__ __attribute__((always_inline)) inline void bring(int step, int i) const {
    const size_t slot = slot_of(step);
    const int stage = step % LATENT_STAGES, lane = made_anew<SHORT>(threadIdx.x) & 63;
    if (i < CODE_LOADS) {
      constexpr int AT_ONCE = 1024 / LATENT;
      const int first = KEYS * half + i * AT_ONCE, key = first + lane / CHUNKS, chunk = (lane ^ (16 * kg + key)) & (CHUNKS - 1);
      lds_dma16_off(uniform_ptr(codes + slot * LATENT), key * LATENT + 16 * chunk, lds_address(&lds.stage[stage].codes[(16 * kg + first) * LATENT]));
    } else if (i < CODE_LOADS + ROPE_LOADS) {
      constexpr int AT_ONCE = 512 / ROPE;
      const int first = (ROPE == 64 ? HALVES == 2 ? half : i - CODE_LOADS : 0) * AT_ONCE, key = first + lane / ROPE_CHUNKS, chunk = (lane ^ key) & (ROPE_CHUNKS - 1);
      lds_dma16_off(uniform_ptr(ropes + slot * ROPE), key * ROPE * 2 + 16 * chunk, lds_address(&lds.stage[stage].ropes[(16 * kg + first) * ROPE * 2]));
    } else if (lane < 4) {                 // (not a load that the compiler waits for: it would wait for the tiles on their way, too)
      lds_dma4_off(uniform_ptr(all_scales + slot), 4 * lane, lds_address(&lds.scales[stage][4 * kg]));
    }
  }
  __device__ __attribute__((always_inline)) inline void bring(int step) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) bring(step, i);
  }
  // scales of keys 4 g .. + 4 of the wave's 16 in a stage; of keys that are not there any, but finite and not zero
  __device__ __attribute__((always_inline)) inline float4_t scales(int stage) const {
    const uint32_t bytes = lds.scales[stage][4 * kg + ((made_anew<SHORT>(threadIdx.x) & 63) >> 4)];
    float4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, (uint32_t)min(max((int)(bytes >> (8 * i) & 255u), 1), 254) << 23);
    return x;
  }
  // zeros for codes that are no numbers, in a tile that has some
  __device__ __attribute__((always_inline)) inline void clean(int stage) const {
    for (int i = threadIdx.x; i < STEP * LATENT / 16; i += 64 * WAVES) {
      u32x4_t w = ((u32x4_t*)lds.stage[stage].codes)[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] &= ~((kv_nan_bytes(w[k]) >> 7) * 0xffu);
      ((u32x4_t*)lds.stage[stage].codes)[i] = w;
    }
  }
};
__device__ inline float latent_exponent(float scale) { return (float)((int)(__builtin_bit_cast(uint32_t, scale) >> 23) - 127); }

// Hides what a row does not see of 16 keys from `key0` on; lane (c, g) has keys 4 g .. + 4 of row c.  odd: no number where a score is none
// before it is hidden (or infinite: no harm)
__device__ __attribute__((always_inline)) inline void latent_mask(float4_t& s, bool there, int key0, int end, int p_row, float& odd) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    odd = __builtin_fmaf(s[i], 0.f, odd);
    const int key = key0 + 4 * g + i;
    if (!there || key >= end || key > p_row) s[i] = -INFINITY;
  }
}

template <int ACT, int LATENT, int ROPE, int RG>
__device__ inline void latent_part(const LatentAttendArgs& args, const KvCrew& crew, const KvPart& pc, const KvRequest& req, LatentLds<LATENT, ROPE, RG>& lds) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  typedef int i32x2_t __attribute__((ext_vector_type(2)));
  using Keys = LatentKeys<LATENT, ROPE, RG>;
  constexpr int WAVES = Keys::WAVES, HALVES = Keys::HALVES, PER = Keys::PER, B = RG / HALVES;        // B: blocks of 16 rows that a wave scores
  constexpr int R = 16 * RG, STEP = LATENT_STEP, CHUNKS = LATENT / 16, ROPE_CHUNKS = ROPE / 8;
  constexpr int LU = LATENT / 64, RU = ROPE / 32, DG = LATENT / 16 / WAVES;
  const AttendArgs& a = args.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
  const int kg = wave & 3, half = wave >> 2;               // the wave's 16 keys of a tile; its half of the rows
  const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0);
  const int i0 = scalar(row0 / a.group), i1 = scalar((row0 + rows - 1) / a.group);
  const int begin = pc.first * STEP, end = min(req.hi(i1), begin + pc.count * STEP);
  const int steps = end > begin ? (end - begin + STEP - 1) / STEP : 0;
  const int p_first = req.p0 + i0;
  const float score_scale = a.scale;

  Keys keys(lds, args, pc, begin, end);
  if (steps > 0) keys.bring(0);
  // The queries: whole rows into the place of the tiles after the first, from there to where each wave multiplies them.  (Each wave
  // reading its own from memory, four waves the same, in pieces of 16 bytes, a part of 64 rows starts 1 to 2 us later.)
  constexpr int KS = 2 * LU + RU, KEPT = KS - latent_queries_in_lds(LATENT, ROPE, RG), ROW = (LATENT + ROPE) / 8, LOADS = (R * ROW + 64 * WAVES - 1) / (64 * WAVES);
  static_assert(R * ROW * 16 <= 2 * sizeof(lds.stage[0]) && ROW % 4 == 0);
  uint8_t* const rows_in = lds.stage[1].codes;             // [row][chunk], chunk c at place c ^ row / 2
  {
    u32x4_t x[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int at = min(tid + 64 * WAVES * j, R * ROW - 1), r = at / ROW, row = min(row0 + r, req.rows - 1), i = row / a.group;
      x[j] = *(const u32x4_t*)(a.q + (size_t)(req.start + i) * a.ldq + (size_t)(row - i * a.group) * (LATENT + ROPE) + 8 * (at - r * ROW));
    }
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int at = min(tid + 64 * WAVES * j, R * ROW - 1), r = at / ROW;        // (the last chunk by several, alike)
      *(u32x4_t*)(rows_in + (r * ROW + ((at - r * ROW) ^ (r >> 1 & 3))) * 16) = x[j];
    }
  }
  __syncthreads();
  u32x4_t q[B][KEPT];
  uint8_t* const q_first = lds.q + ((16 * B * half + c) * 4 + (g ^ (c >> 1 & 3))) * 16;
  const auto q_place = [&](int b, int k) __attribute__((always_inline)) { return q_first + ((k - KEPT) * R + 16 * b) * 64; };
#pragma unroll
  for (int b = 0; b < B; ++b) {
    const uint8_t* const row = rows_in + (16 * (B * half + b) + c) * ROW * 16;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const u32x4_t x = lds_read16(row + ((k < 2 * LU ? 8 * (k >> 1) + 2 * g + (k & 1) : 4 * k + g) ^ (c >> 1 & 3)) * 16);
      if (k < KEPT) q[b][k] = x;
      else if (kg == 0) *(u32x4_t*)q_place(b, k) = x;
    }
  }
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int k = 0; k < KEPT; ++k) asm volatile("" : "+v"(q[b][k]));       // (read before the tiles come)
  __syncthreads();
  if (steps > 1) keys.bring(1);

  float4_t o[DG][RG];
  float m[RG], l[B];
#pragma unroll
  for (int b = 0; b < B; ++b) l[b] = 0.f;
#pragma unroll
  for (int b = 0; b < RG; ++b) {
    m[b] = KV_M_START;
#pragma unroll
    for (int d = 0; d < DG; ++d) o[d][b] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (tid < LATENT_STAGES) lds.odd[tid] = lds.grown[tid] = 0;
  // scores of a tile's keys: lane (c, g) has keys 4 g .. + 4 of row c of each block of rows.  (Two sums of one block in turn: one waits
  // twice as long for itself as an instruction takes.)
  constexpr int SUMS = B == 1 ? 2 : 1;
  float4_t s[B];
  float add[B];                            // to l, once it is settled
  const auto own_reference = [&](int b) __attribute__((always_inline)) { return HALVES == 2 ? half ? m[RG - B + b] : m[b] : m[b]; };
  // the weights of the wave's keys and rows; the largest
  const auto weights = [&](int step, float4_t scale) __attribute__((always_inline)) {
    const float4_t weight_scale = scale * (1.f / LATENT_LIFTED);
    float largest = 0.f;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int row = 16 * (B * half + b) + c;
      const float ref = own_reference(b) - LATENT_LIFT;
      // (l sums up weights of as many bits as are multiplied: of a row that one token rules, their rounding cancels.  What binary16's smallest
      // numbers cut from P besides, 2^21 below the row's largest, stays in l)
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], score_scale, -ref));
      if constexpr (ACT == ACT_F16) {      // (they may lie outside of its range before they are times 2^e)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = latent_round11(p[i]);
        add[b] = (p[0] + p[1]) + (p[2] + p[3]);
      } else add[b] = kv_add2<ACT>(kv_pack<ACT>(p[2], p[3]), kv_add2<ACT>(kv_pack<ACT>(p[0], p[1]), 0.f));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] *= weight_scale[i];
        largest = fmaxf(largest, p[i]);
      }
      *(u32x2_t*)(lds.p[step & 1] + row * (2 * STEP) + (((2 * kg + (g >> 1)) ^ (c & 7)) * 16) + 8 * (g & 1)) = u32x2_t{kv_pack<ACT>(p[0], p[1]), kv_pack<ACT>(p[2], p[3])};
    }
    return largest;
  };
  const auto scores = [&](int step) __attribute__((always_inline)) {
    const int stage = step % LATENT_STAGES, t0 = begin + STEP * step, id = keys.id_of(step);
    const uint8_t* const codes = lds.stage[stage].codes + (16 * kg + c) * LATENT;
    const int chunk0 = made_anew<Keys::SHORT>(g ^ ((16 * kg + c) & (CHUNKS - 1)));
    const uint8_t* const ropes = lds.stage[stage].ropes + (16 * kg + c) * ROPE * 2;
    // Items: the rope part's chunks, then the codes'.  A chunk is read two items ahead of its products, a query that lies in LDS one such query ahead.
    constexpr int T = RU + LU;
    const auto chunk = [&](int t) __attribute__((always_inline)) {
      return t < RU ? lds_read16(ropes + (((4 * t + g) ^ (c & (ROPE_CHUNKS - 1))) * 16)) : lds_read16(codes + ((4 * (t - RU)) ^ chunk0) * 16);
    };
    u32x4_t w[3], qn[2][B];
    const auto fetch = [&](int k) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < B; ++b) qn[k & 1][b] = lds_read16(q_place(b, k));
    };
    // (of units in LDS: KEPT .. KS, the rope part's come first)
    const auto after = [](int k) { return k == KS - 1 ? KEPT : k + 1; };
    const auto unit = [&](int k, u32x4_t key, float4_t (&to)[B]) __attribute__((always_inline)) {
      if (KEPT < KS && k >= KEPT && after(k) != 2 * LU) fetch(after(k));
#pragma unroll
      for (int b = 0; b < B; ++b) to[b] = mfma16<ACT>(key, k < KEPT ? q[b][k < KEPT ? k : 0] : qn[k & 1][b], to[b]);
    };
    static_assert(KEPT == KS || (KEPT <= 2 * LU && (KS - KEPT) % 2 == 0), "every unit's neighbour in the order has the other buffer");
    w[0] = chunk(0);
    w[1] = chunk(1);
    if (KEPT < KS) fetch(2 * LU);
    float4_t x[SUMS][B], y[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      y[b] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < SUMS; ++k) x[k][b] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
    float4_t scale;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (t + 2 < T) w[(t + 2) % 3] = chunk(t + 2);
      else if (t + 2 == T) scale = keys.scales(stage);
      if (t < RU) unit(2 * LU + t, w[t % 3], y);
      else
#pragma unroll
        for (int h = 0; h < 2; ++h) unit(2 * (t - RU) + h, kv_operand<ACT>(w[t % 3][2 * h], w[t % 3][2 * h + 1]), x[h % SUMS]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[b][i] = __builtin_fmaf(SUMS == 2 ? x[0][b][i] + x[SUMS - 1][b][i] : x[0][b][i], scale[i], y[b][i]);
    const bool all_seen = id >= 0 && t0 + STEP <= end && t0 + STEP - 1 <= p_first;
    if (!all_seen) {                       // (rows that all see a code that is no number need no zeros for it)
      float any = 0.f;
#pragma unroll
      for (int b = 0; b < B; ++b)
        latent_mask(s[b], id >= 0, t0 + 16 * kg, end, req.p0 + min(made_anew(row0 + 16 * (B * half + b) + c), req.rows - 1) / a.group, any);
      if (any != any) lds.odd[stage] = 1;
    }
    if (weights(step, scale) > LatentHeld<ACT>::GROWN) lds.grown[stage] = 1;
  };
  // What the barrier behind a tile's scores has made known: where a row of the workgroup has outgrown its reference, all waves find the rows'
  // largest s + e and those rows' weights are made again; a tile with codes that are no numbers is cleaned.
  const auto settle = [&](int step) __attribute__((always_inline)) {
    const int stage = step % LATENT_STAGES;
    const int odd = scalar((int)lds.odd[stage]), grown = scalar((int)lds.grown[stage]);
    if (__builtin_expect(odd | grown, 0)) {
      if (odd) keys.clean(stage);
      if (grown) {
        const float4_t scale = keys.scales(stage);
#pragma unroll
        for (int b = 0; b < B; ++b) {
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, __builtin_fmaf(s[b][i], score_scale, latent_exponent(scale[i])));
          top = max_of_groups(top);
          if (g == 0) ((float*)&lds.most[16 * (B * half + b) + c])[kg] = top;
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < RG; ++b) {
          const float4_t t = lds.most[16 * b + c];
          const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
          const float to = top - m[b] > KV_M_SLACK + 0.0625f + LatentHeld<ACT>::BITS ? top - LatentHeld<ACT>::BITS : m[b], f = __builtin_amdgcn_exp2f(m[b] - to);        // (a row's own: no other row changes its bits)
          m[b] = to;
          if (b / B == half) l[b % B] *= f;
#pragma unroll
          for (int d = 0; d < DG; ++d) o[d][b] *= f;
        }
        weights(step, scale);
      }
      __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < B; ++b) l[b] += add[b];
    if (tid == 0) lds.odd[(step + 2) % LATENT_STAGES] = lds.grown[(step + 2) % LATENT_STAGES] = 0;       // (of the tile before: read by all a barrier ago)
  };

  // One barrier a tile, behind the second product of the tile before, its scores and weights.  Those go by the references so far: what a row's largest
  // s + e has to outgrow them by is seldom (the first tile's always do).
  if (steps > 0) {
    if (steps > 1) vm_wait<PER>();
    else vm_wait<0>();
    __syncthreads();
    scores(0);
    vm_wait<0>();
    __syncthreads();
    settle(0);
  }
  for (int step = 0; step < steps; ++step) {
    const int stage = step % LATENT_STAGES;
    keys.look_ahead(step);
    // dims 16 (DG wave + d) .. of all rows
    if (step + 2 < steps) keys.bring(step + 2);              // (here, where its issue hides behind products)
    const int key0 = made_anew<Keys::SHORT>(8 * g + (c >> 1));
    const uint8_t* const row = lds.stage[stage].codes + key0 * LATENT + 8 * (c & 1);
    const auto values = [&](int n) __attribute__((always_inline)) {        // 32 keys n / DG, 16 dims n % DG
      const int k = n / DG, d = n % DG;
      return __builtin_amdgcn_ds_read_tr8_b64_v2i32(
          (__attribute__((address_space(3))) i32x2_t*)(row + 32 * k * LATENT + (((DG * wave + d) ^ ((32 * k + key0) & (CHUNKS - 1))) * 16)));
    };
    u32x4_t p[RG];
    i32x2_t w[3];
    const uint8_t* const mine = lds.p[step & 1] + c * (2 * STEP);
#pragma unroll
    for (int b = 0; b < RG; ++b) p[b] = lds_read16(mine + 16 * b * (2 * STEP) + ((g ^ (c & 7)) * 16));
    w[0] = values(0);
    w[1] = values(1);
#pragma unroll
    for (int n = 0; n < 2 * DG; ++n) {
      if (n + 2 < 2 * DG) w[(n + 2) % 3] = values(n + 2);
      const u32x4_t v = kv_operand<ACT>((uint32_t)w[n % 3][0], (uint32_t)w[n % 3][1]);
#pragma unroll
      for (int b = 0; b < RG; ++b) o[n % DG][b] = mfma16<ACT>(v, p[b], o[n % DG][b]);
      if (n == DG - 1)
#pragma unroll
        for (int b = 0; b < RG; ++b) p[b] = lds_read16(mine + 16 * b * (2 * STEP) + (((4 + g) ^ (c & 7)) * 16));
      __builtin_amdgcn_sched_barrier(0);
    }
    if (step + 1 < steps) scores(step + 1);
    vm_wait<0>();                          // tile step + 2 has landed, the wave's keys by its own count, the others' by the barrier
    __syncthreads();
    if (step + 1 < steps) settle(step + 1);
  }

  // l of a row: four lanes' keys of four waves
  __syncthreads();
#pragma unroll
  for (int b = 0; b < B; ++b) {
    l[b] += __shfl_xor(l[b], 16, 64);
    l[b] += __shfl_xor(l[b], 32, 64);
    if (g == 0) ((float*)&lds.most[16 * (B * half + b) + c])[kg] = l[b];
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < RG; ++b) {
    const int at = 16 * b + c, row = row0 + at;
    const float4_t t = lds.most[at];
    const float sum = (t[0] + t[1]) + (t[2] + t[3]);
    if (pc.parts > 1) {
      float* const slot = crew.slots + (size_t)pc.slot * latent_stride<LATENT, RG>();
#pragma unroll
      for (int d = 0; d < DG; ++d) *(float4_t*)(slot + (((wave * DG + d) * RG + b) * 64 + lane) * 4) = o[d][b];
      if (wave == 0 && g == 0) {
        slot[R * LATENT + at] = m[b];
        slot[R * (LATENT + 1) + at] = sum;
      }
    } else if (at < rows) {
      const float inv = kv_inverse(sum, a, req, pc.r, row) * LATENT_LIFTED;
      const int i = row / a.group;
      uint16_t* const to = a.out + (size_t)(req.start + i) * a.ldo + (size_t)(row - i * a.group) * LATENT + 4 * g;
#pragma unroll
      for (int d = 0; d < DG; ++d) {
        const float4_t x = o[d][b] * inv;
        *(u32x2_t*)(to + 16 * (DG * wave + d)) = u32x2_t{kv_pack<ACT>(x[0], x[1]), kv_pack<ACT>(x[2], x[3])};
      }
    }
  }
}

}  // namespace glowq
