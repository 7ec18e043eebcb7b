// experts.hip -- routing of tokens to experts, the plan that lays the chosen pairs
// out by expert, and the weighted sum of a token's experts (include/mxq.h states
// them).
#include <type_traits>

#include "mxq_internal.h"

namespace mxq {

namespace {

constexpr int kThreads = 256;

__device__ inline float bf16f(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ inline uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// ---------------------------------------------------------------------------
// Reductions over a wave by DPP moves (a lane without a source takes `none`); the
// result is that of lane 63.

template <int CTRL, int ROWS>
__device__ inline uint32_t dpp_or(uint32_t x, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ inline uint64_t dpp_or(uint64_t x, uint64_t none) {
  return (uint64_t)dpp_or<CTRL, ROWS>((uint32_t)(x >> 32), (uint32_t)(none >> 32)) << 32 |
         dpp_or<CTRL, ROWS>((uint32_t)x, (uint32_t)none);
}
__device__ inline uint32_t last_lane(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ inline uint64_t last_lane(uint64_t x) {
  return (uint64_t)last_lane((uint32_t)(x >> 32)) << 32 | last_lane((uint32_t)x);
}

constexpr int kShr1 = 0x111, kShr2 = 0x112, kShr4 = 0x114, kShr8 = 0x118, kBcast15 = 0x142,
              kBcast31 = 0x143;

template <typename U, typename F>
__device__ inline U wave_reduce(U v, U none, F f) {
  v = f(v, dpp_or<kShr1, 0xF>(v, none));
  v = f(v, dpp_or<kShr2, 0xF>(v, none));
  v = f(v, dpp_or<kShr4, 0xF>(v, none));
  v = f(v, dpp_or<kShr8, 0xF>(v, none));
  v = f(v, dpp_or<kBcast15, 0xA>(v, none));
  v = f(v, dpp_or<kBcast31, 0xC>(v, none));
  return last_lane(v);
}
template <typename U>
__device__ inline U wave_max(U v) {
  return wave_reduce(v, (U)0, [](U a, U b) { return a > b ? a : b; });
}
__device__ inline float wave_sum(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ inline double wave_sum(double v) {
  return __builtin_bit_cast(
      double, wave_reduce(__builtin_bit_cast(uint64_t, v), (uint64_t)0, [](uint64_t a, uint64_t b) {
        return __builtin_bit_cast(uint64_t,
                                  __builtin_bit_cast(double, a) + __builtin_bit_cast(double, b));
      }));
}

// Keys that order as their values do, above 0, which stands for no expert.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);             // (-0 and +0 are equal)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ inline uint64_t key_of(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
  return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}

// A wave per token; lane l holds the scores of experts l, l + 64, ...
template <int NE, bool BIAS>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 64) +
                    __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= a.T) return;
  float x[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = 64 * i + lane;
    x[i] = -__builtin_inff();
    if (e < a.E) {
      const int64_t at = t * a.ld + e;
      const float v = a.logits_f32 ? ((const float *)a.logits)[at]
                                   : bf16f(((const uint16_t *)a.logits)[at]);
      x[i] = v == v ? fminf(v, 3.40282347e38f) : -__builtin_inff();
    }
  }
  const bool softmax = a.score == MXQ_SCORE_SOFTMAX;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const uint32_t k = x[i] == -__builtin_inff() ? 0u : key_of(x[i]);
    top = k > top ? k : top;
  }
  top = wave_max(top);
  const float most = value_of(top);                        // (unused where no expert is left)

  // keys of the choice: the score's, or those of score + bias in 64 bits
  uint64_t key[NE];
  if (BIAS) {
    double s[NE], all = 0.0;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const bool in = x[i] != -__builtin_inff();
      s[i] = !in ? 0.0 : softmax ? exp((double)x[i] - (double)most) : 1.0 / (1.0 + exp(-(double)x[i]));
      all += s[i];
    }
    if (softmax) all = wave_sum(all);
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = 64 * i + lane;
      const double v = (softmax ? s[i] / all : s[i]) + (e < a.E ? (double)a.bias[e] : 0.0);
      key[i] = x[i] == -__builtin_inff() || !(v > -__builtin_inf()) ? 0 : key_of(v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i)                           // (the index below: the lowest wins)
      key[i] = x[i] == -__builtin_inff()
                   ? 0
                   : (uint64_t)key_of(x[i]) << 32 | (uint32_t)~(64 * i + lane);
  }
  int id = -1;                                             // lane j: the j-th choice and its score
  float sc = 0.f;
  for (int j = 0; j < a.k; ++j) {
    uint64_t best = 0;
    int at = 0;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (key[i] > best) {
        best = key[i];
        at = i;
      }
    const uint64_t win = wave_max(best);
    if (win == 0) break;
    int e;
    if (BIAS) {
      const uint32_t mine = best == win ? ~(uint32_t)(64 * at + lane) : 0u;
      e = (int)~wave_max(mine);
    } else {
      e = (int)~(uint32_t)win;
    }
    float xe = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (e >> 6 == i) {
        xe = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x[i]), e & 63));
        if (lane == (e & 63)) key[i] = 0;
      }
    if (lane == j) {
      id = e;
      sc = xe;
    }
  }
  // float64 exponentials of the chosen: x - most is not exact in 32 bits
  double s = 0.0;
  if (id >= 0)
    s = softmax ? exp((double)sc - (double)most) : 1.0 / (1.0 + exp(-(double)sc));
  double sum = 1.0;
  if (a.normalise) {
    sum = wave_sum(s);
  } else if (softmax) {
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      all += x[i] == -__builtin_inff() ? 0.f : expf(x[i] - most);
    sum = (double)wave_sum(all);
  }
  if (lane < a.k) {
    a.ids[t * a.k + lane] = id;
    a.weights[t * a.k + lane] = id >= 0 && sum > 0.0 ? (float)((double)a.scale * (s / sum)) : 0.f;
  }
}

// The plan, a workgroup per expert: the counts of all of them, its own rows.
__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs a) {
  __shared__ int count[kMaxExperts];
  __shared__ int part[kThreads / 64];
  const int t = threadIdx.x, e = blockIdx.x, lane = t & 63, wave = t >> 6;
  for (int i = t; i < a.E; i += kThreads) count[i] = 0;
  __syncthreads();
  for (int64_t p = t; p < a.pairs; p += kThreads) {
    const int id = a.ids[p];
    if (id >= 0 && id < a.E) atomicAdd(&count[id], 1);
  }
  __syncthreads();
  int before = 0;
  for (int i = t; i < e; i += kThreads) before += (count[i] + 15) & ~15;
  before = (int)wave_reduce((uint32_t)before, 0u, [](uint32_t x, uint32_t y) { return x + y; });
  if (lane == 0) part[wave] = before;
  __syncthreads();
  int row = 0;
  for (int w = 0; w < kThreads / 64; ++w) row += part[w];
  const int end = row + ((count[e] + 15) & ~15);
  if (t == 0) a.first[e] = row;
  if (t == 0 && e == a.E - 1) a.first[a.E] = end;
  for (int i = row + count[e] + t; i < end; i += kThreads) a.pair[i] = -1;
  if (e == a.E - 1)
    for (int64_t i = end + t; i < a.rows; i += kThreads) a.pair[i] = -1;
  for (int64_t p0 = 0; p0 < a.pairs; p0 += kThreads) {
    const bool mine = p0 + t < a.pairs && a.ids[p0 + t] == e;
    const uint64_t who = __ballot(mine);
    __syncthreads();
    if (lane == 0) part[wave] = __popcll(who);
    __syncthreads();
    int at = row, all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      at += w < wave ? part[w] : 0;
      all += part[w];
    }
    if (mine) a.pair[at + __popcll(who & (((uint64_t)1 << lane) - 1))] = (int)(p0 + t);
    row += all;
  }
}

// A thread per column of a token.
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.T * a.N) return;
  const int64_t t = i / a.N, c = i - t * a.N;
  float acc = a.residual ? bf16f(a.residual[t * a.ldr + c]) : 0.f;
  for (int64_t j = 0; j < a.k; ++j) {
    const int64_t p = t * a.k + j;
    const int id = a.ids[p];
    if (id < 0 || id >= a.E) continue;
    const int64_t at = p * a.ldy + c;
    const float y = a.y_f32 ? ((const float *)a.y)[at] : bf16f(((const uint16_t *)a.y)[at]);
    acc = fmaf(a.weights[p], y, acc);
  }
  if (a.out_f32) ((float *)a.out)[t * a.ldo + c] = acc;
  else ((uint16_t *)a.out)[t * a.ldo + c] = to_bf16(acc);
}

}  // namespace

hipError_t launch_expert_plan(const PlanArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(plan_kernel, dim3((unsigned)a.E), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_route(const RouteArgs &a, const PlanArgs &p, hipStream_t s) {
  if (a.T > 0) {
    const dim3 grid((unsigned)((a.T + kThreads / 64 - 1) / (kThreads / 64))), block(kThreads);
    auto go = [&](auto ne) {
      constexpr int NE = decltype(ne)::value;
      if (a.bias) hipLaunchKernelGGL((route_kernel<NE, true>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((route_kernel<NE, false>), grid, block, 0, s, a);
    };
    if (a.E <= 64) go(std::integral_constant<int, 1>{});
    else if (a.E <= 128) go(std::integral_constant<int, 2>{});
    else if (a.E <= 256) go(std::integral_constant<int, 4>{});
    else if (a.E <= 512) go(std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 16>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return launch_expert_plan(p, s);
}

hipError_t launch_combine(const CombineArgs &a, hipStream_t s) {
  const int64_t n = (a.T * a.N + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(combine_kernel, dim3((unsigned)n), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace mxq
