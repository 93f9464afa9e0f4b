// Device-side building blocks of rotary positions.
//
// Pair i of a head's rotated dims at position p turns by the angle t = p f_i:
//     (a, b) -> magnitude (a cos t - b sin t, a sin t + b cos t).
// A frequency is kept as a fraction of a whole turn in 64-bit fixed point, F = f / 2 pi * 2^64, so that p F mod 2^64 is the angle,
// reduced exactly at any position; its upper 32 bits leave an error of 2^-32 turns (1.5e-9).  Sine and cosine are summed up
// from their series on an eighth of a turn to either side, to the last bit or so of fp32.  No table is read, and the forty
// instructions of a pair's angle are shared by the heads that a thread takes.
#pragma once
#include "common.hpp"

namespace glowq {

struct RopeView {
  const unsigned long long* turns;     // [rotary_dim / 2]
  int units;                           // rotary_dim / 16: eight pairs each
  int pairs;                           // 0: pair i is dims (i, i + rotary_dim / 2); 1: dims (2 i, 2 i + 1)
  float magnitude;
  // the first of the eight dims that are one half of unit u's vectors, and of the other; units past the rotated ones are 16 dims as
  // they stand
  __device__ inline int dim_a(int u) const { return u >= units || pairs ? 16 * u : 8 * u; }
  __device__ inline int dim_b(int u) const { return u >= units || pairs ? 16 * u + 8 : 8 * (u + units); }
};

__device__ inline void rope_angle(unsigned long long turns, int p, float magnitude, float& c, float& s) {
  const uint32_t x = __umulhi((uint32_t)turns, (uint32_t)p) + (uint32_t)(turns >> 32) * (uint32_t)p;       // of 2^32 a turn
  const uint32_t quarter = (x + 0x20000000u) >> 30;                                // the nearest
  const float r = (float)(int32_t)(x - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32: |r| <= pi / 4
  const float z = r * r;
  // first terms left out: r^11 / 11! < 2e-9, r^12 / 12! < 2e-10
  float sn = __builtin_fmaf(z, 2.7557319223985893e-6f, -1.9841269841269841e-4f);
  sn = __builtin_fmaf(z, sn, 8.3333333333333333e-3f);
  sn = __builtin_fmaf(z, sn, -1.6666666666666667e-1f);
  sn = __builtin_fmaf(r * z, sn, r);
  float cs = __builtin_fmaf(z, -2.7557319223985888e-7f, 2.4801587301587302e-5f);
  cs = __builtin_fmaf(z, cs, -1.3888888888888889e-3f);
  cs = __builtin_fmaf(z, cs, 4.1666666666666667e-2f);
  cs = __builtin_fmaf(z, cs, -0.5f);
  cs = __builtin_fmaf(z, cs, 1.f);
  const float swapped_c = quarter & 1 ? sn : cs, swapped_s = quarter & 1 ? cs : sn;
  c = ((quarter + 1) & 2 ? -swapped_c : swapped_c) * magnitude;
  s = (quarter & 2 ? -swapped_s : swapped_s) * magnitude;
}

// N angles, of pairs from `first` on
template <int N> struct RopeAngles {
  float c[N], s[N];
  __device__ inline void set(const RopeView& r, int first, int p) {
#pragma unroll
    for (int i = 0; i < N; ++i) rope_angle(r.turns[first + i], p, r.magnitude, c[i], s[i]);
  }
};

// (a, b) turned by one angle
__device__ inline void rope_turn(float& a, float& b, float c, float s) {
  const float x = __builtin_fmaf(a, c, -(b * s)), y = __builtin_fmaf(a, s, b * c);
  a = x;
  b = y;
}

// Two vectors turned by N angles: element by element, or each one's neighbours
template <int N> __device__ inline void rope_turn_unit(float (&u)[N], float (&v)[N], const float (&c)[N], const float (&s)[N], bool pairs) {
  if (pairs) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      rope_turn(u[2 * i], u[2 * i + 1], c[i], s[i]);
      rope_turn(v[2 * i], v[2 * i + 1], c[N / 2 + i], s[N / 2 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) rope_turn(u[i], v[i], c[i], s[i]);
  }
}

// 16 bytes of type TYPE (glowq_dtype) at p as fp32, and back with one rounding
template <int TYPE> constexpr int rope_width() { return TYPE == 2 ? 4 : 8; }
template <int TYPE> __device__ inline void rope_load16(const void* p, float (&x)[rope_width<TYPE>()]) {
  if constexpr (TYPE == 2) {
    const float4_t v = *(const float4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  } else if constexpr (TYPE == 0) {
    const half8_t v = *(const half8_t*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  } else {
    const u32x4_t v = *(const u32x4_t*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = v[i];
      x[2 * i] = __builtin_bit_cast(float, w << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
    }
  }
}
template <int TYPE> __device__ inline void rope_store16(void* p, const float (&x)[rope_width<TYPE>()]) {
  if constexpr (TYPE == 2) {
    *(float4_t*)p = float4_t{x[0], x[1], x[2], x[3]};
  } else {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (uint32_t)to_act16<TYPE>(x[2 * i]) | (uint32_t)to_act16<TYPE>(x[2 * i + 1]) << 16;
    *(u32x4_t*)p = v;
  }
}

// Rows of up to four tensors whose heads are rotated together.
constexpr int ROPE_TENSORS = 4;
struct RopeTensor {
  const char* x;
  char* y;
  long long ldx, ldy;          // bytes from row to row
  long long lhx, lhy;          // bytes from head to head
  int end;                     // heads of this tensor and those before it
};
struct RotateArgs {
  RopeView rope;
  RopeTensor t[ROPE_TENSORS];
  const int32_t* positions;
  int T, heads;                // of all tensors
  int units;                   // of a head, two vectors of 16 bytes each
  int groups, per;             // a thread takes heads group, group + groups, ..: `per` at most
};

// Thread `i` of T * groups * units: two vectors of a row, of several heads, with the same angles.  Vectors are 16 bytes whatever the
// type, so that a wave's accesses lie side by side (32 bits with eight numbers a vector: 73 us for 250 MB, 58 so).
template <int TYPE>
__device__ inline void rope_rotate(const RotateArgs& a, long long i) {
  constexpr int SIZE = TYPE == 2 ? 4 : 2, W = rope_width<TYPE>(), PARTS = 8 / W;
  const int at = (int)(i % a.units), unit = at / PARTS, part = at % PARTS;
  const long long j = i / a.units;
  const int group = (int)(j % a.groups);
  const long long row = j / a.groups;
  if (row >= a.T) return;
  const int p = a.positions[row];
  if (p < 0) return;
  const bool turn = unit < a.rope.units;
  const int first = a.rope.dim_a(unit) + (a.rope.pairs ? 2 : 1) * W * part;
  const int da = first * SIZE, db = (a.rope.pairs ? first + W : a.rope.dim_b(unit) + W * part) * SIZE;
  RopeAngles<W> angle;
  if (turn) angle.set(a.rope, 8 * unit + W * part, p);
  for (int h = group; h < a.heads; h += a.groups) {
    int k = 0, before = 0;
#pragma unroll
    for (int n = 0; n < ROPE_TENSORS - 1; ++n)
      if (h >= a.t[n].end) { k = n + 1; before = a.t[n].end; }
    const RopeTensor& t = a.t[k];
    const char* const x = t.x + row * t.ldx + (h - before) * t.lhx;
    char* const y = t.y + row * t.ldy + (h - before) * t.lhy;
    if (!turn && x == y) continue;
    float u[W], v[W];
    rope_load16<TYPE>(x + da, u);
    rope_load16<TYPE>(x + db, v);
    if (turn) rope_turn_unit(u, v, angle.c, angle.s, a.rope.pairs);
    rope_store16<TYPE>(y + da, u);
    rope_store16<TYPE>(y + db, v);
  }
}

}  // namespace glowq
