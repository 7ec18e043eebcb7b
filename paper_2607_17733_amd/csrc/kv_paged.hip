// kv_paged.hip -- new tokens into the paged MXINT KV cache, and rows back out of
// it (include/mxq.h states the pages' layout).
//
// MXSens (arXiv 2607.17733), Appendix A.2: K and V are quantized to MXINT with
// 32-element blocks along the head dimension.  A row of 128 values takes sixteen
// lanes of eight values: a block is four adjacent lanes, whose largest magnitude
// gives the shared exponent; each lane rounds its eight values and packs them,
// 4 bytes of a 4-bit block, 8 of an 8-bit one, neighbours joining what straddles.
// Keys are rotated first, in the lanes that hold them (the partner values of a
// rotation in halves are read a second time, from the cache), and rounded to
// bf16, so that the rows are those of mxq_rope followed by mxq_quantize_rows, bit
// for bit.  The queries of the same tokens are rotated by the same launch.
//
// Bytes bound it.  A workgroup holds sixteen consecutive tokens of one head: in
// a run of tokens each plane of a page is then written in whole runs of 16 times
// 4 m_b bytes.  4001 tokens, 32 query and 8 KV heads, 4/4/6/8 bits, 90 MB: 20 us for
// the rows and the queries together (4.4 TB/s; a large copy moves 4.7).  Read back,
// 10000 rows of 8 heads, 52 MB: 14.5 us; 64 tokens appended: 4.1 us, most of it the
// launch.
#include "mxq_device.h"
#include "mxq_internal.h"
#include "rope_device.h"

namespace mxq {

namespace {

constexpr int kThreads = 256;
constexpr int kLanesPerRow = 16;
constexpr int kTokens = kThreads / kLanesPerRow;
constexpr int kD = 128;

// Eight values (d0 ..) of a row, rotated; `x` is the row.
__device__ inline rope_u4 load_rotated(const RopeArgs &r, const uint16_t *x, int d0, int p) {
  const rope_u4 u = *(const rope_u4 *)(x + d0);
  if (!r.table || d0 >= r.rot) return u;
  if (p < 0 || p >= r.positions) return rope_u4{~0u, ~0u, ~0u, ~0u};
  const float *row = r.table + (int64_t)p * r.rot;
  rope_f4 cs[4];
  if (r.pairs) {
#pragma unroll
    for (int i = 0; i < 2; ++i) cs[i] = *(const rope_f4 *)(row + d0 + 4 * i);
    return rotate_pairs8(u, cs);
  }
  const int half = r.rot / 2;
  const bool second = d0 >= half;
  const int i0 = second ? d0 - half : d0;
#pragma unroll
  for (int i = 0; i < 4; ++i) cs[i] = *(const rope_f4 *)(row + 2 * i0 + 4 * i);
  return rotate_half8(u, *(const rope_u4 *)(x + (second ? i0 : d0 + half)), cs, second);
}

// A lane's eight values as integers: the mantissas of a block of width m and
// exponent E.  The scaled value has at most 8 significant bits, so every step is
// exact but the rounding.
__device__ inline void quantize8(rope_u4 x, int E, int m, bool away, bool full, int (&q)[8]) {
  const float most = (float)((1 << (m - 1)) - 1), least = full ? -most - 1.f : -most;
  const int sh = 127 + m - 2 - E;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = __builtin_amdgcn_ldexpf(
        (i & 1) ? __uint_as_float(x[i >> 1] & 0xFFFF0000u) : bf16_to_f32(x[i >> 1]), sh);
    const float r = away ? __builtin_roundf(v) : __builtin_rintf(v);
    q[i] = E == 255 ? 0 : (int)fminf(fmaxf(r, least), most);
  }
}

// The lane's part of the packed block at p (layout (C) of include/mxq.h); j is
// its place among the block's four lanes, all of which call.
__device__ inline void store_packed(uint8_t *p, int m, int j, const int (&q)[8], bool keep) {
  uint32_t lo = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) lo |= ((uint32_t)q[i] & 15u) << (4 * i);
  if (m == 4) {
    if (keep) *(uint32_t *)(p + 4 * j) = lo;
  } else if (m == 8) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= ((uint32_t)q[i] & 255u) << (8 * (i & 3));
    if (keep) {
      *(uint32_t *)(p + 8 * j) = w[0];
      *(uint32_t *)(p + 8 * j + 4) = w[1];
    }
  } else if (m == 6) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      top |= (((uint32_t)q[i] >> 4) & 3u) << (8 * (i >> 1) + ((j & 1) ? 2 : 6) - 2 * (i & 1));
    top |= (uint32_t)__shfl_xor((int)top, 1);
    if (keep) {
      *(uint32_t *)(p + 4 * j) = lo;
      if (!(j & 1)) *(uint32_t *)(p + 16 + 2 * j) = top;
    }
  } else {
    uint32_t w = 0;                                        // 24 bits; lane j's word takes the next lane's
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= ((uint32_t)q[i] & 7u) << (3 * i);
    const uint32_t next = (uint32_t)__shfl_down((int)w, 1);
    if (keep && j < 3) *(uint32_t *)(p + 4 * j) = (w >> (8 * j)) | (next << (24 - 8 * j));
  }
}

// The lane's eight mantissas back from the packed block.
__device__ inline void load_packed(const uint8_t *p, int m, int j, int (&q)[8]) {
  if (m == 8) {
    const uint32_t w[2] = {*(const uint32_t *)(p + 8 * j), *(const uint32_t *)(p + 8 * j + 4)};
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = sext_bits(w[i >> 2] >> (8 * (i & 3)), 8);
  } else if (m == 4) {
    const uint32_t w = *(const uint32_t *)(p + 4 * j);
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = sext_bits(w >> (4 * i), 4);
  } else if (m == 6) {
    const uint32_t w = *(const uint32_t *)(p + 4 * j);
    const uint32_t top = *(const uint32_t *)(p + 16 + 4 * (j >> 1)) >> ((j & 1) ? 0 : 4);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      q[i] = sext_bits(((w >> (4 * i)) & 15u) | ((top >> (8 * (i >> 1) + 2 - 2 * (i & 1))) & 3u) << 4, 6);
  } else {
    const uint32_t a = p[3 * j] | (uint32_t)p[3 * j + 1] << 8 | (uint32_t)p[3 * j + 2] << 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = sext_bits(a >> (3 * i), 3);
  }
}

// Where a head's rows of a page begin (in units of page_tokens rows).
__device__ inline int64_t page_run(const PageGeo &g, int64_t slot, int head) {
  return ((slot >> g.lg_page) * g.Hkv + head) << g.lg_page;
}

__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvAppendArgs a) {
  const PageGeo &g = a.geo;
  // the heads of sixteen tokens run together: K's, V's, then the queries'
  const uint32_t heads = (uint32_t)(2 * g.Hkv + a.Hq);
  const uint32_t tile = blockIdx.x / heads;
  int head = (int)(blockIdx.x - tile * heads);
  const int lane = threadIdx.x % kLanesPerRow, d0 = 8 * lane;
  const int64_t row = (int64_t)tile * kTokens + threadIdx.x / kLanesPerRow;
  const bool in = row < a.T;                               // (every lane takes part in the exchanges)
  const int64_t t = in ? row : a.T - 1;
  const int pos = a.rope.table ? a.pos[t] : 0;
  if (head >= 2 * g.Hkv) {
    head -= (int)(2 * g.Hkv);
    const rope_u4 x = load_rotated(a.rope, a.q + t * a.q_ts + head * a.q_hs, d0, pos);
    // (in place, a row's lanes have all read, their partners' values too, before one writes)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (in) *(rope_u4 *)(a.q_out + (t * a.Hq + head) * kD + d0) = x;
    return;
  }
  const bool is_v = head >= g.Hkv;
  if (is_v) head -= (int)g.Hkv;
  const int64_t slot = a.slots[t];
  const bool keep = in && slot >= 0 && slot < g.pages << g.lg_page;
  RopeArgs none = a.rope;
  if (is_v) none.table = nullptr;
  const rope_u4 x = load_rotated(none, is_v ? a.v + t * a.v_ts + head * a.v_hs
                                            : a.k + t * a.k_ts + head * a.k_hs, d0, pos);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = x[i] & 0x7FFF7FFFu;
    top = max(top, max(u & 0xFFFFu, u >> 16));
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  const int E = block_exponent(top);
  const int b = lane >> 2, j = lane & 3;
  const int m = b == 0 ? g.m[0] : b == 1 ? g.m[1] : b == 2 ? g.m[2] : g.m[3];
  const int off = b == 0 ? g.off[0] : b == 1 ? g.off[1] : b == 2 ? g.off[2] : g.off[3];
  int q[8];
  quantize8(x, E, m, a.ties_away, a.full_clamp, q);
  const int64_t base = page_run(g, keep ? slot : 0, head);
  const int i = (int)((keep ? slot : 0) & ((1 << g.lg_page) - 1));
  uint8_t *mant = (is_v ? a.v_mant : a.k_mant) + base * g.row + ((int64_t)off << g.lg_page) +
                  (int64_t)i * 4 * m;
  store_packed(mant, m, j, q, keep);
  uint32_t ex = (uint32_t)E << (8 * b);
  ex |= (uint32_t)__shfl_xor((int)ex, 4);
  ex |= (uint32_t)__shfl_xor((int)ex, 8);
  if (keep && lane == 0) *(uint32_t *)((is_v ? a.v_exp : a.k_exp) + (base + i) * 4) = ex;
}

__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvReadArgs a) {
  const PageGeo &g = a.geo;
  const uint32_t heads = (uint32_t)((a.k ? g.Hkv : 0) + (a.v ? g.Hkv : 0));
  const uint32_t tile = blockIdx.x / heads;
  int head = (int)(blockIdx.x - tile * heads);
  const int64_t t = (int64_t)tile * kTokens + threadIdx.x / kLanesPerRow;
  if (t >= a.n) return;
  const bool is_v = !a.k || head >= g.Hkv;
  if (a.k && is_v) head -= (int)g.Hkv;
  const int lane = threadIdx.x % kLanesPerRow, b = lane >> 2, j = lane & 3;
  const int64_t slot = a.slots[t];
  rope_u4 y = {0u, 0u, 0u, 0u};
  if (slot >= 0 && slot < g.pages << g.lg_page) {
    const int m = b == 0 ? g.m[0] : b == 1 ? g.m[1] : b == 2 ? g.m[2] : g.m[3];
    const int off = b == 0 ? g.off[0] : b == 1 ? g.off[1] : b == 2 ? g.off[2] : g.off[3];
    const int64_t base = page_run(g, slot, head);
    const int i = (int)(slot & ((1 << g.lg_page) - 1));
    const uint8_t *mant = (is_v ? a.v_mant : a.k_mant) + base * g.row +
                          ((int64_t)off << g.lg_page) + (int64_t)i * 4 * m;
    int q[8];
    load_packed(mant, m, j, q);
    const int sh = (int)(is_v ? a.v_exp : a.k_exp)[(base + i) * 4 + b] - 127 - (m - 2);
    // exact, at most 8 significant bits, but for -2^128 (the full clamp's lowest mantissa with
    // E = 254), which is out of bf16's range: its lowest value, not an infinity
    auto value = [&](int i) {
      return f32_to_bf16(fmaxf(__builtin_amdgcn_ldexpf((float)q[i], sh), -0x1.FEp127f));
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = value(2 * k) | value(2 * k + 1) << 16;
  }
  *(rope_u4 *)((is_v ? a.v : a.k) + (t * g.Hkv + head) * kD + 8 * lane) = y;
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs &a, hipStream_t s) {
  const int64_t n = (a.T + kTokens - 1) / kTokens * (2 * a.geo.Hkv + a.Hq);
  hipLaunchKernelGGL(kv_append_kernel, dim3((unsigned)n), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvReadArgs &a, hipStream_t s) {
  const int64_t n = (a.n + kTokens - 1) / kTokens * ((a.k ? a.geo.Hkv : 0) + (a.v ? a.geo.Hkv : 0));
  hipLaunchKernelGGL(kv_read_kernel, dim3((unsigned)n), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace mxq
