// Attention over rows of keys and values (latent attention, expanded): a head's keys are its own numbers beside a part that all heads
// share, values have as many numbers as the former.
//
// A workgroup takes 128 rows of one head of a request, 32 to a wave, and a part of the keys (kv_cut), 64 a step.  Keys, their
// shared part and values lie in LDS as they come, brought by direct loads a tile ahead, 16-byte chunks of a row permuted by its key so
// that the reads of a wave meet all banks.  As for the cache of keys and values scores come transposed, S^T = K Q^T (32x32x16), and the weights
// are the second product's operand, O^T = V^T P^T, as they stand: V's operand comes transposed out of LDS, four keys of 16 dims at a
// time, in the order of keys that the scores have.  l sums up the rounded weights.  In binary16 a row's largest weight is 2^7 to 2^15, the upper
// end of the type, so that something of what is 2^31 below it is left (100000 keys behind one that weighs 2^22, 2^24 or 2^26 of theirs and whose
// value is zero: error 2.6e-4, 2.6e-4, 8.3e-4 of the output; with 2^0 to 2^8 it was 3.7e-3, 2e-2, 1).
//
// Bound.  A prompt of 8000 tokens, 32 heads of 128 + 64, bfloat16: 0.61 ms, 1.07 PFLOP/s, two workgroups on a CU, the matrix pipe busy 0.6 of the
// time at the 1.7 GHz that the machine keeps under it.  Each of four waves reads a whole tile of 41 KB for its 40 products, which
// LDS takes as long for as the products last; reads go two products ahead (765 us without), places are worked out
// once for both stages, and the queries are waited for before the loop (their count in it would be one of tiles on their way: 947 us
// with four-byte reads).
#pragma once
#include "kv_attend.hpp"
#include "wide.hpp"

namespace glowq {

constexpr int EXPANDED_WAVES = 4, EXPANDED_THREADS = 64 * EXPANDED_WAVES, EXPANDED_ROWS = 32 * EXPANDED_WAVES, EXPANDED_STEP = 64, EXPANDED_STAGES = 2;

struct ExpandedArgs {
  AttendArgs a;                // kv_heads = heads, group = 1
  const uint16_t *k, *r, *v;
  const int32_t* key_starts;
  long long lhq;
  int ldk, lhk, ldr, ldv, lhv;
  int keys;
};

template <int N, int ROPE> struct alignas(16) ExpandedStage {
  uint8_t k[EXPANDED_STEP * N * 2], r[EXPANDED_STEP * ROPE * 2], v[EXPANDED_STEP * N * 2];
};
template <int N, int ROPE> struct ExpandedLds {
  union {
    ExpandedStage<N, ROPE> stage[EXPANDED_STAGES];
    uint32_t flags[2];         // behind the keys: a result that is no number; a value that is none
  };
};

template <int ACT>
__device__ inline float16_t expanded_mfma(u32x4_t a, u32x4_t b, float16_t c) {
  if constexpr (ACT == ACT_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Where chunk c of key's row lies: of rows of CHUNKS chunks that are read a chunk a key, and of values
template <int CHUNKS> __device__ inline int key_chunk(int c, int key) { return CHUNKS == 4 ? c ^ ((key >> 1) & 3) : c ^ (key % CHUNKS); }
template <int CHUNKS> __device__ inline int value_chunk(int c, int key) {
  return CHUNKS == 16 ? c ^ ((key & 3) << 2 | ((key >> 2) & 3)) : c ^ ((key & 1) << 2 | ((key >> 1) & 3));
}

// A row's largest weight is 2^BITS where its reference is new, and 2^KV_M_SLACK of that at most.
template <int ACT> struct ExpandedHeld { static constexpr float BITS = ACT == ACT_F16 ? 7.f : 0.f; };

template <int V> struct ExpandedNumber { static constexpr int VALUE = V; };

// both halves of a word, zeros for those that are infinities or NaN
template <int ACT> __device__ inline uint32_t finite_halves(uint32_t w) {
  constexpr uint32_t INF = ACT == ACT_F16 ? 0x7c00u : 0x7f80u;
  if ((w & INF) == INF) w &= 0xffff0000u;
  if ((w >> 16 & INF) == INF) w &= 0xffffu;
  return w;
}

// 1 / l of a finished row: zeros for one that sees no key, NaN for one whose keys all score -infinity
__device__ inline float expanded_inverse(float l, const KvRequest& q, int row) { return l != 0.f ? 1.f / l : q.hi(row) > 0 ? NAN : 0.f; }

// The request's keys lie in rows first ..; it has no more than there are behind that
__device__ inline int expanded_keys(const ExpandedArgs& x, int r, KvRequest& req) {
  const int first = min(max(x.key_starts[r], 0), x.keys);
  req.len = min(req.len, x.keys - first);
  return first;
}

template <int ACT, int N, int ROPE>
__device__ inline void expanded_part(const ExpandedArgs& x, const KvCrew& crew, const KvPart& pc, KvRequest& req, ExpandedLds<N, ROPE>& lds) {
  constexpr int R = EXPANDED_ROWS, STEP = EXPANDED_STEP, C = N / 8, RC = ROPE / 8, NB = N / 32;
  typedef short short4_t __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, hf = lane >> 5;
  const int key0 = __builtin_amdgcn_readfirstlane(expanded_keys(x, pc.r, req));
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0), first = row0 + 32 * wave;
  const int begin = pc.first * STEP, end = min(req.hi(row0 + rows - 1), begin + pc.count * STEP);
  const int steps = end > begin ? (end - begin + STEP - 1) / STEP : 0;
  const bool any_row = first < req.rows;
  const int p_row = req.p0 + first + c32, p_first = req.p0 + first, p_last = req.p0 + min(first + 31, req.rows - 1);

  u32x4_t q[(N + ROPE) / 16];
  {
    const int row = min(first + c32, req.rows - 1);
    const uint16_t* const src = a.q + (size_t)(req.start + row) * a.ldq + pc.head * x.lhq + 8 * hf;
#pragma unroll
    for (int u = 0; u < (N + ROPE) / 16; ++u) q[u] = *(const u32x4_t*)(src + 16 * u);
  }
  // (the queries have come before loads into LDS begin: those are waited for by their number)
#pragma unroll
  for (int u = 0; u < (N + ROPE) / 16; ++u) asm volatile("" : "+v"(q[u]));
  const uint16_t* const kh = uniform_ptr(x.k + (size_t)key0 * x.ldk + (size_t)pc.head * x.lhk);
  const uint16_t* const rh = uniform_ptr(x.r + (size_t)key0 * x.ldr);
  const uint16_t* const vh = uniform_ptr(x.v + (size_t)key0 * x.ldv + (size_t)pc.head * x.lhv);

  // The wave's 16 keys of a tile, a load 64 chunks; keys behind the request's last are that one again (whole tiles need neither
  // the comparison nor a product for every load: these were a fifth of the vector ALU's work)
  const auto bring = [&](int step) __attribute__((always_inline)) {
    const int t0 = begin + STEP * step, most = min(req.len - 1 - t0, STEP - 1);
    ExpandedStage<N, ROPE>& to = lds.stage[step % EXPANDED_STAGES];
    const auto load = [&](const uint16_t* rows, int ld, auto CHUNKS, auto place, uint8_t* there) __attribute__((always_inline)) {
      constexpr int CH = decltype(CHUNKS)::VALUE, KEYS = 64 / CH;
      const uint16_t* const tile = uniform_ptr(rows + (size_t)t0 * ld);
#pragma unroll
      for (int i = 0; i < 16 / KEYS; ++i) {
        const int key = 16 * wave + i * KEYS + lane / CH, at = i * KEYS * CH * 16;
        const uint32_t chunk = 16 * place(lane % CH, key);
        if (most == STEP - 1) lds_dma16_off(uniform_ptr(tile + (uint32_t)((16 * wave + i * KEYS) * ld)), (uint32_t)(lane / CH * ld) * 2 + chunk, lds_address(there + at));
        else lds_dma16_off(tile, (uint32_t)(min(key, most) * ld) * 2 + chunk, lds_address(there + at));
      }
    };
    load(kh, x.ldk, ExpandedNumber<C>{}, [](int c, int key) { return key_chunk<C>(c, key); }, to.k + 16 * wave * N * 2);
    load(vh, x.ldv, ExpandedNumber<C>{}, [](int c, int key) { return value_chunk<C>(c, key); }, to.v + 16 * wave * N * 2);
    load(rh, x.ldr, ExpandedNumber<RC>{}, [](int c, int key) { return key_chunk<RC>(c, key); }, to.r + 16 * wave * ROPE * 2);
  };
  // Where the wave reads in stage 0: what differs by the key's place in 16 or by the chunk; all else, the stage too, goes into the instructions
  const uint8_t *k_at[N / 16], *r_at[ROPE / 16], *v_at[2][NB];
#pragma unroll
  for (int u = 0; u < N / 16; ++u) k_at[u] = lds.stage[0].k + c32 * N * 2 + 16 * key_chunk<C>(2 * u + hf, c32);
#pragma unroll
  for (int u = 0; u < ROPE / 16; ++u) r_at[u] = lds.stage[0].r + c32 * ROPE * 2 + 16 * key_chunk<RC>(2 * u + hf, c32);
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int key = 8 * y + 4 * hf + ((lane & 15) >> 2), chunk = 4 * j + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      v_at[y][j] = lds.stage[0].v + key * N * 2 + 16 * value_chunk<C>(chunk, key) + 8 * (lane & 1);
    }

  float16_t o[NB];
  float m, l;
  bool found = false;
  const auto tile = [&](auto AGAIN, auto STAGE, int step) __attribute__((always_inline)) {
    constexpr int FROM = decltype(STAGE)::VALUE * (int)sizeof(ExpandedStage<N, ROPE>);
    const int t0 = begin + STEP * step;
    // (reads go two products' time ahead of what takes them)
    constexpr int U = (N + ROPE) / 16;
    const auto keys = [&](int u, int kb) __attribute__((always_inline)) {
      return u < N / 16 ? *(const u32x4_t*)(k_at[u] + FROM + kb * 32 * N * 2) : *(const u32x4_t*)(r_at[u - N / 16] + FROM + kb * 32 * ROPE * 2);
    };
    float16_t s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
    u32x4_t k[3][2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) k[u][kb] = keys(u, kb);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u + 2 < U)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) k[(u + 2) % 3][kb] = keys(u + 2, kb);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = expanded_mfma<ACT>(k[u % 3][kb], q[u], s[kb]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!(t0 + STEP - 1 <= p_first && t0 + STEP <= end)) {
      const int most = min(end - 1, p_row);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (t0 + 32 * kb + 8 * (e >> 2) + 4 * hf + (e & 3) > most) s[kb][e] = -INFINITY;
    }
    float most = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) most = fmaxf(most, s[kb][e]);
    most *= a.scale;
    constexpr float HELD = ExpandedHeld<ACT>::BITS;
    if (__any(most > m + (KV_M_SLACK + HELD))) {
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      const float to = most > m + (KV_M_SLACK + HELD) ? most - HELD : m, f = __builtin_amdgcn_exp2f(m - to);        // (a row's own: no other row changes its bits)
      m = to;
      l *= f;
#pragma unroll
      for (int j = 0; j < NB; ++j) o[j] *= f;
    }
    // V's operand n: keys 16 (n / NB) + 4 hf .. + 4 and 8 further, dims 32 (n % NB) ..
    const auto values = [&](int n) __attribute__((always_inline)) {
      u32x4_t w;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const u32x2_t t = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(v_at[y][n % NB] + FROM + n / NB * 16 * N * 2)));
        w[2 * y] = t[0];
        w[2 * y + 1] = t[1];
      }
      return w;
    };
    constexpr int AHEAD = 3;
    u32x4_t v[AHEAD + 1];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) v[n] = values(n);
    u32x4_t p[4];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h >> 1][8 * (h & 1) + 2 * i], a.scale, -m));
        const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h >> 1][8 * (h & 1) + 2 * i + 1], a.scale, -m));
        p[h][i] = kv_pack<ACT>(e0, e1);
        l = kv_add2<ACT>(p[h][i], l);
      }
#pragma unroll
    for (int n = 0; n < 4 * NB; ++n) {
      if (n + AHEAD < 4 * NB) v[(n + AHEAD) % (AHEAD + 1)] = values(n + AHEAD);
      u32x4_t w = v[n % (AHEAD + 1)];
      if constexpr (decltype(AGAIN)::VALUE)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = finite_halves<ACT>(w[i]);
          found = found || x != w[i];
          w[i] = x;
        }
      o[n % NB] = expanded_mfma<ACT>(w, p[n / NB], o[n % NB]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  const auto pass = [&](auto AGAIN) __attribute__((always_inline)) {
    m = KV_M_START;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][e] = 0.f;
    if (steps > 0) bring(0);
    const auto half = [&](auto STAGE, int step) __attribute__((always_inline)) {
      // this tile has landed, the wave's keys by its own count, the others' by the barrier; and everyone is done with the one before
      vm_wait<0>();
      __syncthreads();
      if (step + 1 < steps) bring(step + 1);
      // (waves whose rows see none of these keys, or that have no rows, only bring theirs)
      if (any_row && begin + STEP * step <= p_last) tile(AGAIN, STAGE, step);
    };
    for (int step = 0; step < steps; step += EXPANDED_STAGES) {
      half(ExpandedNumber<0>{}, step);
      if (step + 1 < steps) half(ExpandedNumber<1>{}, step + 1);
    }
  };
  pass(ExpandedNumber<0>{});
  // 0 * NaN or infinity of a value that other rows see has reached rows that do not: then a second pass, zeros for such values
  float any = 0.f;
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) any = __builtin_fmaf(o[j][e], 0.f, any);
  __syncthreads();                         // (the tiles are done with)
  if (tid == 0) lds.flags[0] = 0;
  __syncthreads();
  if (any != any && first + c32 < req.rows) lds.flags[0] = 1;
  __syncthreads();
  if (lds.flags[0]) {
    __syncthreads();                       // (all have looked: LDS is free)
    pass(ExpandedNumber<1>{});
  }
  if (__any(found) && any_row) {
    // the rows that do see such values get them: every dim of every key of the part is looked at
    for (int key = begin; key < end; ++key) {
      if (key > p_row) continue;
      const uint16_t* const row = vh + (size_t)key * x.ldv;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint32_t w = row[32 * j + 8 * (e >> 2) + 4 * hf + (e & 3)];
          constexpr uint32_t INF = ACT == ACT_F16 ? 0x7c00u : 0x7f80u;
          if ((w & INF) == INF) o[j][e] += kv_act_f32<ACT>(w);
        }
    }
  }

  const int at = 32 * wave + c32, row = row0 + at;
  const float sum = l + __shfl_xor(l, 32, 64);
  if (pc.parts > 1) {
    if (!any_row) return;
    float* const slot = crew.slots + (size_t)pc.slot * (R * (N + 2));
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *(float4_t*)(slot + (((wave * NB + j) * 4 + e / 4) * 64 + lane) * 4) = float4_t{o[j][e], o[j][e + 1], o[j][e + 2], o[j][e + 3]};
    if (hf == 0) {
      slot[R * N + at] = m;
      slot[R * (N + 1) + at] = sum;
    }
    return;
  }
  const float inv = expanded_inverse(sum, req, row);
  uint16_t* const to = a.out + (size_t)(req.start + row) * a.ldo + (size_t)pc.head * N;
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int e = 0; e < 16; e += 8) {
      // elements e .. e + 3 are dims base + 4 hf .. + 4, the next four 8 further; lanes 32 apart exchange halves: eight dims in
      // a row each
      const int base = 32 * j + 2 * e;
      const float4_t y = float4_t{o[j][e], o[j][e + 1], o[j][e + 2], o[j][e + 3]} * inv;
      const float4_t z = float4_t{o[j][e + 4], o[j][e + 5], o[j][e + 6], o[j][e + 7]} * inv;
      const auto lo = __builtin_amdgcn_permlane32_swap(kv_pack<ACT>(y[0], y[1]), kv_pack<ACT>(z[0], z[1]), false, false);
      const auto hi = __builtin_amdgcn_permlane32_swap(kv_pack<ACT>(y[2], y[3]), kv_pack<ACT>(z[2], z[3]), false, false);
      if (at < rows) *(u32x4_t*)(to + base + 8 * hf) = u32x4_t{lo[0], hi[0], lo[1], hi[1]};
    }
}

}  // namespace glowq
