// rope.hip -- rotary positions on bf16 rows: the table of cosines and sines, and
// the rotation (include/mxq.h states both).
//
// The pair (x1, x2) of frequency f at position p turns by the angle p f:
// (x1 c - x2 s, x2 c + x1 s).  The angle is taken in float64, where p f is exact
// to 2^-53 of itself: at position 2^20 that is 1e-10 of a turn, where float32
// would be 0.06 off.  So the table is built once, and the rotation is one pass
// over the rows: bytes bound it, 2 D read and 2 D written per head, the table's
// row shared by a token's heads.  4096 tokens of 32 heads, half of each head rotated,
// 68 MB: 12.5 us (5.4 TB/s; a plain copy of far more moves 4.7); one token: 2.4 us,
// most of it the launch.
#include "mxq_internal.h"
#include "rope_device.h"

namespace mxq {

namespace {

constexpr int kThreads = 256;

struct Freqs {
  double f[kRopeMaxRot / 2];
};

__global__ __launch_bounds__(kThreads) void rope_table_kernel(Freqs fr, int half, int64_t n,
                                                              double mscale, float *table) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t p = i / half;
  double s, c;
  sincos((double)p * fr.f[i - p * half], &s, &c);
  table[2 * i] = (float)(mscale * c);
  table[2 * i + 1] = (float)(mscale * s);
}

// One thread per sixteen values of a rotation in halves (eight and their
// partners), per eight of a rotation in pairs or of the part that is copied.
__global__ __launch_bounds__(kThreads) void rope_vec_kernel(RopeRowsArgs a, uint32_t per_head,
                                                            uint32_t rot_items, int64_t total) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (id >= total) return;
  const uint32_t per_token = per_head * (uint32_t)a.H;
  const int64_t t = id / per_token;
  const uint32_t r = (uint32_t)(id - t * per_token), h = r / per_head, e = r - h * per_head;
  const uint16_t *x = a.x + t * a.x_ts + h * a.x_hs;
  uint16_t *y = a.y + t * a.y_ts + h * a.y_hs;
  const int rot = a.rope.rot;
  if (e >= rot_items) {
    const uint32_t d = rot + 8 * (e - rot_items);
    *(rope_u4 *)(y + d) = *(const rope_u4 *)(x + d);
    return;
  }
  const int p = a.pos[t];
  const bool out = p < 0 || p >= a.rope.positions;
  const float *row = a.rope.table + (int64_t)(out ? 0 : p) * rot;
  rope_f4 cs[4];
  if (a.rope.pairs) {
#pragma unroll
    for (int i = 0; i < 2; ++i) cs[i] = *(const rope_f4 *)(row + 8 * e + 4 * i);
    const rope_u4 v = rotate_pairs8(*(const rope_u4 *)(x + 8 * e), cs);
    *(rope_u4 *)(y + 8 * e) = out ? rope_u4{~0u, ~0u, ~0u, ~0u} : v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = *(const rope_f4 *)(row + 16 * e + 4 * i);
    const rope_u4 u = *(const rope_u4 *)(x + 8 * e), v = *(const rope_u4 *)(x + rot / 2 + 8 * e);
    const rope_u4 nan = {~0u, ~0u, ~0u, ~0u};
    *(rope_u4 *)(y + 8 * e) = out ? nan : rotate_half8(u, v, cs, false);
    *(rope_u4 *)(y + rot / 2 + 8 * e) = out ? nan : rotate_half8(v, u, cs, true);
  }
}

// Rows whose sizes or strides rule the 16-byte accesses out: one thread per pair
// of values.
__global__ __launch_bounds__(kThreads) void rope_any_kernel(RopeRowsArgs a, int64_t total) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (id >= total) return;
  const int64_t per_head = a.D / 2, per_token = per_head * a.H;
  const int64_t t = id / per_token, r = id - t * per_token, h = r / per_head;
  const int e = (int)(r - h * per_head), rot = a.rope.rot, half = rot / 2;
  const uint16_t *x = a.x + t * a.x_ts + h * a.x_hs;
  uint16_t *y = a.y + t * a.y_ts + h * a.y_hs;
  if (e >= half) {
    y[2 * e] = x[2 * e];
    y[2 * e + 1] = x[2 * e + 1];
    return;
  }
  const int i = a.rope.pairs ? 2 * e : e, j = a.rope.pairs ? 2 * e + 1 : e + half;
  const int p = a.pos[t];
  if (p < 0 || p >= a.rope.positions) {
    y[i] = y[j] = 0xFFFF;
    return;
  }
  const float *row = a.rope.table + (int64_t)p * rot + 2 * e;
  const float u = bf16_to_f32(x[i]), v = bf16_to_f32(x[j]);
  y[i] = (uint16_t)f32_to_bf16(rotated(u, v, row[0], row[1], false));
  y[j] = (uint16_t)f32_to_bf16(rotated(v, u, row[0], row[1], true));
}

}  // namespace

hipError_t launch_rope_table(const double *inv_freq, int rot, int64_t positions, double mscale,
                             float *table, hipStream_t s) {
  Freqs fr;
  for (int i = 0; i < rot / 2; ++i) fr.f[i] = inv_freq[i];
  for (int i = rot / 2; i < kRopeMaxRot / 2; ++i) fr.f[i] = 0.0;
  const int64_t n = positions * (rot / 2);
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)),
                     dim3(kThreads), 0, s, fr, rot / 2, n, mscale, table);
  return hipGetLastError();
}

hipError_t launch_rope(const RopeRowsArgs &a, hipStream_t s) {
  const int rot = a.rope.rot;
  const bool vec = a.D % 8 == 0 && rot % (a.rope.pairs ? 8 : 16) == 0 &&
                   (a.x_ts | a.x_hs | a.y_ts | a.y_hs) % 8 == 0 &&
                   (((uintptr_t)a.x | (uintptr_t)a.y) & 15) == 0;
  auto grid = [](int64_t n) { return dim3((unsigned)((n + kThreads - 1) / kThreads)); };
  if (vec) {
    const uint32_t rot_items = (uint32_t)(rot / (a.rope.pairs ? 8 : 16));
    // (in place, what is not rotated is there already)
    const uint32_t per_head = rot_items + (a.x == a.y ? 0u : (uint32_t)((a.D - rot) / 8));
    const int64_t n = a.T * a.H * per_head;
    hipLaunchKernelGGL(rope_vec_kernel, grid(n), dim3(kThreads), 0, s, a, per_head, rot_items, n);
  } else {
    const int64_t n = a.T * a.H * (a.D / 2);
    hipLaunchKernelGGL(rope_any_kernel, grid(n), dim3(kThreads), 0, s, a, n);
  }
  return hipGetLastError();
}

}  // namespace mxq
