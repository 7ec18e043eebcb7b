// rope_device.h -- the rotation of rotary positions, shared by the kernels that
// rotate rows (rope.hip) and those that rotate keys on their way into the cache
// (kv_paged.hip): the same operations in the same order, so that both give the
// same bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mxq_internal.h"

namespace mxq {

typedef unsigned rope_u4 __attribute__((ext_vector_type(4)));
typedef float rope_f4 __attribute__((ext_vector_type(4)));

__device__ inline float bf16_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ inline uint32_t f32_to_bf16(float x) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
}

// a * c - b * s (SIGN > 0: a * c + b * s), every operation rounded on its own.
__device__ inline float rotated(float a, float b, float c, float s, bool plus) {
#pragma clang fp contract(off)
  const float x = a * c, y = b * s;
  return plus ? x + y : x - y;
}

// Eight values of the first half (plus false) or the second half (plus true) of
// a rotation in halves: x the values, p their partners, cs the pairs (c, s).
__device__ inline rope_u4 rotate_half8(rope_u4 x, rope_u4 p, const rope_f4 (&cs)[4], bool plus) {
  rope_u4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = rotated(bf16_to_f32(x[i]), bf16_to_f32(p[i]), cs[i][0], cs[i][1], plus);
    const float hi = rotated(__uint_as_float(x[i] & 0xFFFF0000u),
                             __uint_as_float(p[i] & 0xFFFF0000u), cs[i][2], cs[i][3], plus);
    y[i] = f32_to_bf16(lo) | f32_to_bf16(hi) << 16;
  }
  return y;
}

// Eight values, four adjacent pairs; cs[0], cs[1] hold their (c, s).
__device__ inline rope_u4 rotate_pairs8(rope_u4 x, const rope_f4 (&cs)[4]) {
  rope_u4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = bf16_to_f32(x[i]), b = __uint_as_float(x[i] & 0xFFFF0000u);
    const float c = cs[i >> 1][2 * (i & 1)], s = cs[i >> 1][2 * (i & 1) + 1];
    y[i] = f32_to_bf16(rotated(a, b, c, s, false)) | f32_to_bf16(rotated(b, a, c, s, true)) << 16;
  }
  return y;
}

struct rope_f8 {
  float v[8];
};
__device__ inline rope_u4 to_bf16x8(const rope_f8 &x) {
  rope_u4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = f32_to_bf16(x.v[2 * i]) | f32_to_bf16(x.v[2 * i + 1]) << 16;
  return y;
}
__device__ inline rope_f8 rotate_half8(const rope_f8 &x, const rope_f8 &p, const rope_f4 (&cs)[4],
                                       bool plus) {
  rope_f8 y;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    y.v[i] = rotated(x.v[i], p.v[i], cs[i >> 1][2 * (i & 1)], cs[i >> 1][2 * (i & 1) + 1], plus);
  return y;
}
__device__ inline rope_f8 rotate_pairs8(const rope_f8 &x, const rope_f4 (&cs)[4]) {
  rope_f8 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x.v[2 * i], b = x.v[2 * i + 1];
    const float c = cs[i >> 1][2 * (i & 1)], s = cs[i >> 1][2 * (i & 1) + 1];
    y.v[2 * i] = rotated(a, b, c, s, false);
    y.v[2 * i + 1] = rotated(b, a, c, s, true);
  }
  return y;
}
// The sum over the n lanes of a head (a power of two), the same in each.
template <int CTRL>
__device__ inline float lane_dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF,
                                                            0xF, false));
}
__device__ inline float sum_lanes(float v, int n) {
  if (n > 1) v += lane_dpp<0xB1>(v);                       // the other of two,
  if (n > 2) v += lane_dpp<0x4E>(v);                       // the other two of four,
  if (n > 4) v += lane_dpp<0x141>(v);                      // four of eight,
  if (n > 8) v += lane_dpp<0x140>(v);                      // eight of sixteen
  if (n > 16) v += __shfl_xor(v, 16);
  if (n > 32) v += __shfl_xor(v, 32);
  return v;
}
__device__ inline double sum_lanes(double v, int n) {
  for (int i = 1; i < n; i *= 2) v += __shfl_xor(v, i);
  return v;
}

// 1 / sqrt(mean of the squares + eps) of a head, from the squares that each of its n
// lanes has added up; f(T) adds the lane's own in T.  In float32 where the sum and eps are
// far from its limits (float64 for all heads made the arithmetic the bound: 4001 tokens of
// 48 heads 24 -> 22 us), else in float64: a head of zeros has no direction, and stays
// zero.
struct HeadNorm {
  float r;
  double wide;             // in r's place where it is not 0
};
template <typename F>
__device__ inline HeadNorm head_norm(F f, int n, int D, float eps) {
  const float s = sum_lanes(f(0.f), n);
  HeadNorm h = {0.f, 0.0};
  if (s > 0x1p-80f && s < 0x1p120f && eps < 0x1p120f) {
    h.r = __builtin_amdgcn_rsqf(fmaf(s, 1.f / (float)D, eps));
  } else {                                                 // (all lanes of the head)
    const double m = sum_lanes(f(0.0), n) / (double)D + (double)eps;
    h.wide = m == 0.0 ? 0.0 : 1.0 / sqrt(m);
  }
  return h;
}
// float32(float32(x r) gain).
__device__ inline float normalised1(float x, const HeadNorm &h, float gain) {
#pragma clang fp contract(off)
  return (h.wide == 0.0 ? x * h.r : (float)((double)x * h.wide)) * gain;
}
__device__ inline rope_f8 normalised8(rope_u4 x, const HeadNorm &h, rope_u4 gain) {
  rope_f8 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y.v[2 * i] = normalised1(bf16_to_f32(x[i]), h, bf16_to_f32(gain[i]));
    y.v[2 * i + 1] = normalised1(__uint_as_float(x[i] & 0xFFFF0000u), h,
                                 __uint_as_float(gain[i] & 0xFFFF0000u));
  }
  return y;
}

// Values d0 .. d0 + 7 of a head of D values at x, normalised and rotated, in one of the
// n lanes (a power of two) that hold it; all n call, `in` those with values.
__device__ inline rope_u4 load_normalised_rotated(const RopeArgs &rope, int p, const uint16_t *x,
                                                  const uint16_t *gain, float eps, int D, int d0,
                                                  int n, bool in) {
  rope_u4 u = {0u, 0u, 0u, 0u}, g = u;
  if (in) {
    u = *(const rope_u4 *)(x + d0);
    g = *(const rope_u4 *)(gain + d0);
  }
  const int rot = rope.rot, half = rot / 2;
  const bool turns = in && d0 < rot, out = p < 0 || p >= rope.positions;
  const bool second = d0 >= half;
  const int i0 = second ? d0 - half : d0;                  // (of a rotation in halves)
  rope_f4 cs[4] = {};
  rope_u4 pu = u, pg = g;
  if (turns) {
    const float *row = rope.table + (int64_t)(out ? 0 : p) * rot;
    if (rope.pairs) {
#pragma unroll
      for (int i = 0; i < 2; ++i) cs[i] = *(const rope_f4 *)(row + d0 + 4 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) cs[i] = *(const rope_f4 *)(row + 2 * i0 + 4 * i);
      const int partner = second ? i0 : d0 + half;
      pu = *(const rope_u4 *)(x + partner);
      pg = *(const rope_u4 *)(gain + partner);
    }
  }
  const HeadNorm r = head_norm(
      [&](auto s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const decltype(s) a = bf16_to_f32(u[i]), b = __uint_as_float(u[i] & 0xFFFF0000u);
          s = fma(a, a, s);
          s = fma(b, b, s);
        }
        return s;
      },
      n, D, eps);
  const rope_f8 v = normalised8(u, r, g);
  if (!turns) return to_bf16x8(v);
  if (out) return rope_u4{~0u, ~0u, ~0u, ~0u};
  if (rope.pairs) return to_bf16x8(rotate_pairs8(v, cs));
  return to_bf16x8(rotate_half8(v, normalised8(pu, r, pg), cs, second));
}

}  // namespace mxq
