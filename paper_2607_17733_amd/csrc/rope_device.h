// rope_device.h -- the rotation of rotary positions, shared by the kernels that
// rotate rows (rope.hip) and those that rotate keys on their way into the cache
// (kv_paged.hip): the same operations in the same order, so that both give the
// same bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

}  // namespace mxq
