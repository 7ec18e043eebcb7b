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

// Queries and keys normalised per head and rotated: L lanes of eight values hold a
// head (a power of two, so that their sum is an exchange within the wave), the
// queries' heads before the keys'.  The values stay in registers between the two;
// those of the partners of a rotation in halves are read again, from the cache.  Bytes
// and vector instructions bound it alike: 4001 tokens of 48 heads, half of each rotated, 99
// MB 21.5 us (4.6 TB/s; a large copy moves 4.7 to 5.2), and 280 instructions to a wave, which
// the SIMDs issue in as long; one token 3 us, the launch.
__global__ __launch_bounds__(kThreads) void rope_qk_kernel(RopeQkArgs a, int lg_lanes,
                                                           int64_t total) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int d0 = 8 * (int)(id & ((1 << lg_lanes) - 1));
  const int64_t head = id >> lg_lanes;
  const bool in = head < total && d0 < a.D;                // (every lane takes part in the sum)
  const uint32_t heads = (uint32_t)(a.Hq + a.Hk);
  const int64_t t = (in ? head : 0) / heads;
  const int h = (int)((in ? head : 0) - t * heads);
  const bool is_k = h >= a.Hq;
  const uint16_t *x = is_k ? a.k + t * a.k_ts + (h - a.Hq) * a.k_hs : a.q + t * a.q_ts + h * a.q_hs;
  uint16_t *y = is_k ? a.k_out + t * a.ko_ts + (h - a.Hq) * a.ko_hs
                     : a.q_out + t * a.qo_ts + h * a.qo_hs;
  const rope_u4 v = load_normalised_rotated(a.rope, a.pos[t], x, is_k ? a.norm.k_gain : a.norm.q_gain,
                                            a.norm.eps, (int)a.D, d0, 1 << lg_lanes, in);
  // (in place, a head's lanes have all read, their partners' values too, before one writes)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (in) *(rope_u4 *)(y + d0) = v;
}

// Heads whose sizes or strides rule the 16-byte accesses out: a wave per head, the
// squares added in the same order.
__global__ __launch_bounds__(kThreads) void rope_qk_any_kernel(RopeQkArgs a, int64_t total) {
  const int lane = threadIdx.x & 63;
  const int64_t head = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (head >= total) return;
  const int64_t heads = a.Hq + a.Hk, t = head / heads;
  const int h = (int)(head - t * heads);
  const bool is_k = h >= a.Hq;
  const uint16_t *x = is_k ? a.k + t * a.k_ts + (h - a.Hq) * a.k_hs : a.q + t * a.q_ts + h * a.q_hs;
  uint16_t *y = is_k ? a.k_out + t * a.ko_ts + (h - a.Hq) * a.ko_hs
                     : a.q_out + t * a.qo_ts + h * a.qo_hs;
  const uint16_t *gain = is_k ? a.norm.k_gain : a.norm.q_gain;
  const int D = (int)a.D, rot = a.rope.rot, half = rot / 2;
  const HeadNorm r = head_norm(
      [&](auto s) {
        for (int c = 8 * lane; c < D; c += 512)
          for (int d = c; d < min(c + 8, D); ++d) {
            const decltype(s) v = bf16_to_f32(x[d]);
            s = fma(v, v, s);
          }
        return s;
      },
      64, D, a.norm.eps);
  auto value = [&](int d) { return normalised1(bf16_to_f32(x[d]), r, bf16_to_f32(gain[d])); };
  const int p = a.pos[t];
  const bool out = p < 0 || p >= a.rope.positions;
  const float *row = a.rope.table + (int64_t)(out ? 0 : p) * rot;
  for (int e = lane; e < half + (D - rot); e += 64) {
    if (e >= half) {
      const int d = rot + e - half;
      y[d] = (uint16_t)f32_to_bf16(value(d));
      continue;
    }
    const int i = a.rope.pairs ? 2 * e : e, j = a.rope.pairs ? 2 * e + 1 : e + half;
    const float u = value(i), v = value(j);
    y[i] = out ? 0xFFFF : (uint16_t)f32_to_bf16(rotated(u, v, row[2 * e], row[2 * e + 1], false));
    y[j] = out ? 0xFFFF : (uint16_t)f32_to_bf16(rotated(v, u, row[2 * e], row[2 * e + 1], true));
  }
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

hipError_t launch_rope_qk(const RopeQkArgs &a, hipStream_t s) {
  const int rot = a.rope.rot;
  const int64_t total = a.T * (a.Hq + a.Hk);
  const int64_t strides = (a.Hq ? a.q_ts | a.q_hs | a.qo_ts | a.qo_hs : 0) |
                          (a.Hk ? a.k_ts | a.k_hs | a.ko_ts | a.ko_hs : 0);
  const uintptr_t at = (a.Hq ? (uintptr_t)a.q | (uintptr_t)a.q_out : 0) |
                       (a.Hk ? (uintptr_t)a.k | (uintptr_t)a.k_out : 0);
  if (a.D % 8 == 0 && a.D <= 512 && rot % (a.rope.pairs ? 8 : 16) == 0 && strides % 8 == 0 &&
      (at & 15) == 0) {
    int lg = 0;
    while (8 << lg < a.D) ++lg;
    hipLaunchKernelGGL(rope_qk_kernel, dim3((unsigned)(((total << lg) + kThreads - 1) / kThreads)),
                       dim3(kThreads), 0, s, a, lg, total);
  } else {
    constexpr int per = kThreads / 64;
    hipLaunchKernelGGL(rope_qk_any_kernel, dim3((unsigned)((total + per - 1) / per)), dim3(kThreads),
                       0, s, a, total);
  }
  return hipGetLastError();
}

}  // namespace mxq
