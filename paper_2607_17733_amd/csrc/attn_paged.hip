// attn_paged.hip -- attention of new tokens over the paged MXINT KV cache
// (include/mxq.h states the operation).
//
// One wave per (query token, query head), two values per lane, one key at a time
// with a running maximum and sum: the plainest form that covers every case.
#include "mxq_device.h"
#include "mxq_internal.h"

namespace mxq {

namespace {

constexpr int kD = 128;

__device__ inline float bf16f(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// Two values (d, d + 1) of a cached row.
__device__ inline float2 cached2(const PageGeo &g, const uint8_t *mant, const uint8_t *exp,
                                 int64_t run, int i, int d) {
  const int b = d >> 5;
  const int m = g.m[b], off = g.off[b];
  const uint8_t *p = mant + run * g.row + ((int64_t)off << g.lg_page) + (int64_t)i * 4 * m;
  const BlockInfo bi{m, 0};
  const int sh = (int)exp[(run + i) * 4 + b] - 127 - (m - 2);
  return float2{__builtin_amdgcn_ldexpf((float)act_elem(p, bi, d & 31), sh),
                __builtin_amdgcn_ldexpf((float)act_elem(p, bi, (d & 31) + 1), sh)};
}

__global__ __launch_bounds__(64) void attn_paged_kernel(AttnPagedArgs a) {
  const PageGeo &g = a.geo;
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, d = 2 * lane;
  int s = 0;
  while (s < a.S && t >= a.cu_q[s + 1]) ++s;
  if (s == a.S || t < a.cu_q[s]) return;
  const int n = a.cu_q[s + 1] - a.cu_q[s];
  int64_t len = a.kv_len[s];
  if (len > a.max_kv) len = a.max_kv;
  if (len > a.table_pages << g.lg_page) len = a.table_pages << g.lg_page;
  const int64_t p = len - n + (t - a.cu_q[s]);
  const int64_t pre = a.prefix ? a.prefix[s] : 0;
  const uint16_t *q = a.q + (int64_t)t * a.q_ts + h * a.q_hs + d;
  const float q0 = bf16f(q[0]), q1 = bf16f(q[1]);
  float m = -__builtin_inff(), l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int64_t j = 0; j < len; ++j) {
    const bool see = (j <= p && (a.window == 0 || p - j < a.window)) || j < pre;
    if (!see) continue;
    const int page = a.table[s * a.ld_table + (j >> g.lg_page)];
    const bool hole = page < 0 || page >= g.pages;
    const int64_t run = ((int64_t)(hole ? 0 : page) * g.Hkv + h / a.G) << g.lg_page;
    const int i = (int)(j & ((1 << g.lg_page) - 1));
    float2 k = cached2(g, a.k_mant, a.k_exp, run, i, d);
    float2 v = cached2(g, a.v_mant, a.v_exp, run, i, d);
    if (hole) k = v = float2{0.f, 0.f};
    float x = q0 * k.x + q1 * k.y;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) x += __shfl_xor(x, w);
    x *= a.scale;
    if (a.softcap > 0.f) x = a.softcap * tanhf(x / a.softcap);
    if (a.slopes) x -= a.slopes[h] * fabsf((float)(p - j));
    const float nm = fmaxf(m, x);
    const float ref = nm == -__builtin_inff() ? 0.f : nm;
    const float f = expf(m - ref), e = expf(x - ref);
    l = l * f + e;
    o0 = o0 * f + e * v.x;
    o1 = o1 * f + e * v.y;
    m = nm;
  }
  const float r = l == 0.f ? 0.f : 1.f / l;
  const int64_t at = ((int64_t)t * a.Hq + h) * kD + d;
  if (a.o_f32) {
    ((float *)a.o)[at] = o0 * r;
    ((float *)a.o)[at + 1] = o1 * r;
  } else {
    ((__bf16 *)a.o)[at] = (__bf16)(o0 * r);
    ((__bf16 *)a.o)[at + 1] = (__bf16)(o1 * r);
  }
}

}  // namespace

int64_t attn_paged_work(const AttnPagedArgs &) { return 0; }

hipError_t launch_attn_paged(const AttnPagedArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(attn_paged_kernel, dim3((unsigned)a.T, (unsigned)a.Hq), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace mxq
