// experts.hip -- routing of tokens to experts, the plan that lays the chosen pairs
// out by expert, and the weighted sum of a token's experts (include/mxq.h states
// them).
//
// Routing.  Both scores rise with the logits, so the choice needs no exponential, only
// an order: a wave holds a token's logits as integer keys, a few to a lane, and takes
// the largest k times by a reduction over the lanes.  The exponentials of the k chosen
// are taken relative to the largest (of the chosen, where only their ratios count).
// With a bias the order is that of score + bias, whose neighbours 32 bits cannot always
// tell apart; 64 bits decide then.  Vector instructions bound it: 8191 tokens among 256
// experts, 8 chosen, with a bias 14 us, 9 of them their issue, without 8 (bytes: 2); one
// token, with its plan by the same workgroup, 3.6, most of it the launch.
//
// Plan.  A counting sort, stable, whole numbers only: 65528 pairs 7 + 2 to 4 us, latency
// (0.5 MB).  Image rows come in sixteens, so an expert wastes 8 rows on average.
//
// Weighted sum.  Bytes: 2048 tokens of 6 experts, 2048 columns, float32 rows 118 MB 23 us
// (5.1 TB/s), bf16 rows 67 MB 13.
#include <algorithm>
#include <type_traits>

#include "mxq_internal.h"

namespace mxq {

namespace {

constexpr int kThreads = 256;

typedef unsigned comb_u4 __attribute__((ext_vector_type(4)));
typedef float comb_f4 __attribute__((ext_vector_type(4)));

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
// The sum over the lanes up to this one.
__device__ inline int lanes_upto(int v) {
  v += (int)dpp_or<kShr1, 0xF>((uint32_t)v, 0u);
  v += (int)dpp_or<kShr2, 0xF>((uint32_t)v, 0u);
  v += (int)dpp_or<kShr4, 0xF>((uint32_t)v, 0u);
  v += (int)dpp_or<kShr8, 0xF>((uint32_t)v, 0u);
  v += (int)dpp_or<kBcast15, 0xA>((uint32_t)v, 0u);
  return v + (int)dpp_or<kBcast31, 0xC>((uint32_t)v, 0u);
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

// The keys of a wave's experts, lane l's being those of l, l + 64, ...; take() gives the
// largest that is left and the lowest expert that has it.  Up to four a lane are put in
// order once, so that a round looks at one of each lane (a round that looked through four
// took 100 instructions: 8191 tokens among 256 experts 15.5 us, ordered 14).
template <int NE, typename U>
struct Keys {
  static constexpr bool kOrdered = NE <= 4;
  U key[NE];
  int at[NE];
  __device__ void order(int lane) {
#pragma unroll
    for (int i = 0; i < NE; ++i) at[i] = 64 * i + lane;
    if (!kOrdered) return;
#pragma unroll
    for (int n = NE - 1; n > 0; --n)                       // (equal ones stay in order)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const bool swap = key[i + 1] > key[i];
        const U k = key[i];
        const int a = at[i];
        key[i] = swap ? key[i + 1] : k;
        at[i] = swap ? at[i + 1] : a;
        key[i + 1] = swap ? k : key[i + 1];
        at[i + 1] = swap ? a : at[i + 1];
      }
  }
  __device__ U take(int &e) {
    U mine = key[0];
    int who = at[0];
    if (!kOrdered) {
#pragma unroll
      for (int i = 1; i < NE; ++i)
        if (key[i] > mine) {
          mine = key[i];
          who = at[i];
        }
    }
    const U win = wave_max(mine);
    const uint64_t lanes = __ballot(mine == win);
    e = __builtin_amdgcn_readlane(who, __builtin_ctzll(lanes));
    if (lanes & (lanes - 1)) e = (int)~wave_max(mine == win ? ~(uint32_t)who : 0u);
    if (kOrdered) {
      const bool out = who == e;
#pragma unroll
      for (int i = 0; i + 1 < NE; ++i) {
        key[i] = out ? key[i + 1] : key[i];
        at[i] = out ? at[i + 1] : at[i];
      }
      key[NE - 1] = out ? 0 : key[NE - 1];
    } else {
#pragma unroll
      for (int i = 0; i < NE; ++i) key[i] = at[i] == e ? 0 : key[i];
    }
    return win;
  }
};

// The choice of one token by one wave; lane l holds the scores of experts l, l + 64,
// ...  Lane j < k returns the j-th choice and its weight.
template <int NE, bool BIAS>
__device__ inline void choose(const RouteArgs &a, int64_t t, int &chosen, float &weight) {
  const int lane = threadIdx.x & 63;
  // (all loads at once, without a branch about them)
  float x[NE], bias[NE];
  const int64_t row = t * a.ld;
  if (a.logits_f32) {
#pragma unroll
    for (int i = 0; i < NE; ++i) x[i] = ((const float *)a.logits)[row + min(64 * i + lane, a.E - 1)];
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i)
      x[i] = bf16f(((const uint16_t *)a.logits)[row + min(64 * i + lane, a.E - 1)]);
  }
  if (BIAS)
#pragma unroll
    for (int i = 0; i < NE; ++i) bias[i] = a.bias[min(64 * i + lane, a.E - 1)];
#pragma unroll
  for (int i = 0; i < NE; ++i)
    x[i] = 64 * i + lane < a.E && x[i] == x[i] ? fminf(x[i], 3.40282347e38f) : -__builtin_inff();
  const bool softmax = a.score == MXQ_SCORE_SOFTMAX;
  Keys<NE, uint32_t> keys;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    keys.key[i] = x[i] == -__builtin_inff() ? 0u : key_of(x[i]);
    top = max(top, keys.key[i]);
  }
  const float most = value_of(wave_max(top));              // (unused where no expert is left)

  int id = -1;                                             // lane j: the j-th choice and its score
  float sc = 0.f;
  if (!BIAS) {
    keys.order(lane);
    for (int j = 0; j < a.k; ++j) {
      int e;
      const uint32_t best = keys.take(e);
      if (best == 0) break;
      if (lane == j) {
        id = e;
        sc = value_of(best);
      }
    }
  } else {
    // The scores in 32 bits first.  Theirs and their sums' errors are below 2^-19 of the
    // larger of 1 and the sum; where two neighbours of the order are within 2^-17, all are
    // formed in 64 bits.
    float s[NE], all = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      s[i] = x[i] == -__builtin_inff() ? 0.f : softmax ? expf(x[i] - most) : 1.f / (1.f + expf(-x[i]));
      all += s[i];
    }
    if (softmax) all = wave_sum(all);
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const float v = (softmax ? s[i] / all : s[i]) + bias[i];
      keys.key[i] = x[i] == -__builtin_inff() || !(v > -__builtin_inff()) ? 0u : key_of(v);
    }
    keys.order(lane);
    float value = 0.f;                                     // lane j: the j-th sum, j <= k
    int found = 0;
    for (int j = 0; j <= a.k; ++j) {
      int e;
      const uint32_t best = keys.take(e);
      if (best == 0) break;
      ++found;
      if (lane == j) {
        value = value_of(best);
        id = e;
      }
    }
    if (lane >= a.k) id = -1;
    const float next = __shfl_down(value, 1);
    const bool near = __ballot(lane + 1 < found &&
                               !(value - next > 0x1p-17f * fmaxf(1.f, fabsf(value)))) != 0;
    if (near) {
      double d[NE], sum = 0.0;
      Keys<NE, uint64_t> wide;
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        d[i] = x[i] == -__builtin_inff() ? 0.0
               : softmax                 ? exp((double)x[i] - (double)most)
                                         : 1.0 / (1.0 + exp(-(double)x[i]));
        sum += d[i];
      }
      if (softmax) sum = wave_sum(sum);
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        const double v = (softmax ? d[i] / sum : d[i]) + (double)bias[i];
        wide.key[i] = x[i] == -__builtin_inff() || !(v > -__builtin_inf()) ? 0 : key_of(v);
      }
      wide.order(lane);
      id = -1;
      for (int j = 0; j < a.k; ++j) {
        int e;
        if (wide.take(e) == 0) break;
        if (lane == j) id = e;
      }
    }
    if (id >= 0) {
      const int64_t at = t * a.ld + id;
      sc = fminf(a.logits_f32 ? ((const float *)a.logits)[at]
                              : bf16f(((const uint16_t *)a.logits)[at]),
                 3.40282347e38f);
    }
  }
  // The chosen scores, relative to exp(ref) where only their ratios count, so that none is
  // lost; x - ref with what its rounding leaves, so that the exponential is good to its
  // own two units.
  float ref = softmax ? most : 0.f;
  if (a.normalise) {
    const float best = value_of(wave_max(id >= 0 ? key_of(sc) : 0u));
    ref = softmax ? best : fminf(best, 0.f);
  }
  // A score below e^-80, soon no normal float32, is held as s e^-88, since a large scale
  // may make a normal weight of it.
  constexpr float kHalf = 7.78113224e-20f;                 // e^-44
  float s = 0.f;
  bool far = false;
  if (id >= 0) {
    const float d = sc - ref, back = d - sc;
    const float rest = (sc - (d - back)) - (ref + back);
    far = d < -80.f;
    // (no scale brings back what lies below -177; far below, d overflows and has no rest)
    s = d < -200.f ? 0.f : expf(far ? d + 88.f : d) * (1.f + rest);
    if (!softmax) s = sc > 0.f ? 1.f / (1.f + expf(-sc)) : s / (1.f + expf(sc));
  }
  float sum = 1.f;
  if (a.normalise) {
    sum = wave_sum(far ? 0.f : s);                         // (the best is not far from itself)
  } else if (softmax) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) sum += x[i] == -__builtin_inff() ? 0.f : expf(x[i] - most);
    sum = wave_sum(sum);
  }
  chosen = id;
  weight = id >= 0 && sum > 0.f ? (far ? a.scale * kHalf * (s / sum) * kHalf : a.scale * (s / sum)) : 0.f;
}

// A wave per token.
template <int NE, bool BIAS>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 64) +
                    __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= a.T) return;
  int id;
  float w;
  choose<NE, BIAS>(a, t, id, w);
  if (lane < a.k) {
    a.ids[t * a.k + lane] = id;
    a.weights[t * a.k + lane] = w;
  }
}

// ---------------------------------------------------------------------------
// The plan, a sort of the pairs by expert that keeps their order: the pairs in at most
// kPlanParts runs, a workgroup each.  One launch counts every run's pairs by expert,
// the next adds the counts up and places the runs' pairs; a single run counts itself.
// 65528 pairs of 256 experts: 7 + 2 to 4 us; with a workgroup to each expert that looked
// through all pairs, in one launch, 20.

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
static_assert(kPlanThreads >= kMaxExperts, "a thread per expert");

// The rows of the experts before this thread's, of which `mine` are its own; last: of
// all of them.  Every thread of the workgroup calls it; part[] is its scratch.
__device__ inline int rows_before(int mine, int *part, int &last) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = lanes_upto(mine);
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  last = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    upto += w < wave ? part[w] : 0;
    last += part[w];
  }
  return upto - mine;
}

__device__ inline int run_of(const PlanArgs &a, int parts) {
  return (int)(((a.pairs + parts - 1) / parts + kPlanThreads - 1) / kPlanThreads) * kPlanThreads;
}
// The pairs of run b by expert into count[], which is zero.
__device__ inline void count_run(const PlanArgs &a, int run, int b, int *count) {
  const int64_t end = min(a.pairs, (int64_t)(b + 1) * run);
  for (int64_t p = (int64_t)b * run + threadIdx.x; p < end; p += kPlanThreads) {
    const int id = a.ids[p];
    if ((unsigned)id < (unsigned)a.E) atomicAdd(&count[id], 1);
  }
}

__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(PlanArgs a) {
  __shared__ int count[kMaxExperts];
  const int t = threadIdx.x, b = blockIdx.x;
  count[t] = 0;
  __syncthreads();
  count_run(a, run_of(a, gridDim.x), b, count);
  __syncthreads();
  if (t < a.E) a.work[b * a.E + t] = count[t];
}

__global__ __launch_bounds__(kPlanThreads) void plan_place_kernel(PlanArgs a) {
  __shared__ int next[kMaxExperts];                        // the row of the run's next pair
  __shared__ uint8_t in_wave[kPlanWaves][kMaxExperts];     // pairs of an expert in a wave
  __shared__ int part[kPlanWaves];
  const int t = threadIdx.x, lane = t & 63, b = blockIdx.x, parts = gridDim.x;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int run = run_of(a, parts);
  int all = 0, before = 0;
  if (parts == 1) {
    next[t] = 0;
    __syncthreads();
    count_run(a, run, 0, next);
    __syncthreads();
    all = next[t];
  } else if (t < a.E) {
    constexpr int kAhead = 16;
    for (int i0 = 0; i0 < parts; i0 += kAhead) {
      int n[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) n[i] = i0 + i < parts ? a.work[(i0 + i) * a.E + t] : 0;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        all += n[i];
        before += i0 + i < b ? n[i] : 0;
      }
    }
  }
  int last;
  const int row = rows_before((all + 15) & ~15, part, last);
  if (t < a.E && t % parts == b)                           // the rows that fill an expert's sixteen
    for (int i = all; i & 15; ++i) a.pair[row + i] = -1;
  if (b == 0 && t < a.E) a.first[t] = row;
  if (b == 0 && t == 0) a.first[a.E] = last;
  for (int64_t i = last + (int64_t)b * kPlanThreads + t; i < a.rows; i += (int64_t)parts * kPlanThreads)
    a.pair[i] = -1;
  next[t] = row + before;

  for (int64_t p0 = (int64_t)b * run; p0 < min(a.pairs, (int64_t)(b + 1) * run); p0 += kPlanThreads) {
    const int64_t p = p0 + t;
    int id = p < a.pairs ? a.ids[p] : -1;
    if ((unsigned)id >= (unsigned)a.E) id = kMaxExperts;   // (a group of its own)
    for (int e = lane; e < a.E; e += 64) in_wave[wave][e] = 0;
    // the lanes of the same expert, bit by bit of its number
    uint64_t same = ~(uint64_t)0;
#pragma unroll
    for (int bit = 0; bit < 11; ++bit) {
      const uint64_t set = __ballot(id >> bit & 1);
      same &= id >> bit & 1 ? set : ~set;
    }
    const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
    if (rank == 0 && id < a.E) in_wave[wave][id] = (uint8_t)__popcll(same);
    __syncthreads();
    if (id < a.E) {
      int at = next[id] + rank;
      for (int w = 0; w < wave; ++w) at += in_wave[w][id];
      a.pair[at] = (int)p;
    }
    __syncthreads();
    if (t < a.E) {                                         // the next thousand's
      int n = 0;
#pragma unroll
      for (int w = 0; w < kPlanWaves; ++w) n += in_wave[w][t];
      next[t] += n;
    }
    __syncthreads();
  }
}

// A few tokens: one workgroup chooses and plans, its pairs and rows in LDS.
constexpr int kFewPairs = 256;

template <int NE, bool BIAS>
__global__ __launch_bounds__(kPlanThreads) void route_few_kernel(RouteArgs a, PlanArgs b) {
  __shared__ int count[kMaxExperts];
  __shared__ int start[kMaxExperts];
  __shared__ int part[kPlanWaves];
  __shared__ __attribute__((aligned(16))) int ids[kFewPairs + 4];
  __shared__ int rows[16 * kFewPairs];
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  for (int i = t; i < a.E; i += kPlanThreads) count[i] = 0;
  for (int i = t; i < (int)b.rows; i += kPlanThreads) rows[i] = -1;
  if (t < 4) ids[(b.pairs & ~3) + t] = -1;                 // (the last four's, before theirs are chosen)
  __syncthreads();
  for (int k = wave; k < (int)a.T; k += kPlanWaves) {
    int id;
    float w;
    choose<NE, BIAS>(a, k, id, w);
    if (lane < a.k) {
      const int p = k * a.k + lane;
      a.ids[p] = id;
      a.weights[p] = w;
      ids[p] = id;
    }
  }
  __syncthreads();
  const int P = (int)b.pairs, id = t < P ? ids[t] : -1;
  int rank = 0;
  if (id >= 0) {
    atomicAdd(&count[id], 1);
#pragma unroll 8
    for (int p = 0; p < P; p += 4) {
      const int4 q = *(const int4 *)(ids + p);
      rank += (p < t && q.x == id) + (p + 1 < t && q.y == id) + (p + 2 < t && q.z == id) +
              (p + 3 < t && q.w == id);
    }
  }
  __syncthreads();
  // an expert's first row: the sums over the experts, a thread to each
  int last;
  const int row = rows_before(t < a.E ? (count[t] + 15) & ~15 : 0, part, last);
  if (t < a.E) {
    start[t] = row;
    b.first[t] = row;
  }
  if (t == 0) b.first[a.E] = last;
  __syncthreads();
  if (id >= 0) rows[start[id] + rank] = t;
  __syncthreads();
  for (int i = t; i < (int)b.rows; i += kPlanThreads) b.pair[i] = rows[i];
}

// ---------------------------------------------------------------------------
// A token's weighted sum: bytes bound it, so eight columns to a thread where the rows
// allow 16-byte pieces, and the loads of four experts' rows in flight.

template <bool VEC>
__device__ inline void combine(const CombineArgs &a, int64_t t, int64_t c) {
  constexpr int C = VEC ? 8 : 1;
  auto unpack = [](comb_u4 v, float *f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(v[e] << 16);
      f[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
    }
  };
  float acc[C] = {};
  if (a.residual) {
    const uint16_t *r = a.residual + t * a.ldr + c;
    if constexpr (VEC) unpack(*(const comb_u4 *)r, acc);
    else acc[0] = bf16f(*r);
  }
  for (int j0 = 0; j0 < (int)a.k; j0 += 4) {
    int id[4];
    float w[4];
    comb_u4 y[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      id[j] = -1;
      if (j0 + j < a.k) {
        const int64_t p = t * a.k + j0 + j;
        id[j] = a.ids[p];
        w[j] = a.weights[p];
        const int64_t at = p * a.ldy + c;
        if constexpr (VEC) {
          const char *row = (const char *)a.y + at * (a.y_f32 ? 4 : 2);
          y[j][0] = *(const comb_u4 *)row;
          if (a.y_f32) y[j][1] = *(const comb_u4 *)(row + 16);
        } else {
          y[j][0][0] = a.y_f32 ? ((const uint32_t *)a.y)[at]
                               : (uint32_t)((const uint16_t *)a.y)[at] << 16;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (id[j] < 0 || id[j] >= a.E) continue;
      float v[C];
      if constexpr (!VEC) {
        v[0] = __uint_as_float(y[j][0][0]);
      } else if (a.y_f32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(y[j][e >> 2][e & 3]);
      } else {
        unpack(y[j][0], v);
      }
#pragma unroll
      for (int e = 0; e < C; ++e) acc[e] = fmaf(w[j], v[e], acc[e]);
    }
  }
  if constexpr (!VEC) {
    if (a.out_f32) ((float *)a.out)[t * a.ldo + c] = acc[0];
    else ((uint16_t *)a.out)[t * a.ldo + c] = to_bf16(acc[0]);
  } else if (a.out_f32) {
    comb_f4 *o = (comb_f4 *)((float *)a.out + t * a.ldo + c);
    o[0] = comb_f4{acc[0], acc[1], acc[2], acc[3]};
    o[1] = comb_f4{acc[4], acc[5], acc[6], acc[7]};
  } else {
    comb_u4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = (uint32_t)to_bf16(acc[2 * e]) | (uint32_t)to_bf16(acc[2 * e + 1]) << 16;
    *(comb_u4 *)((uint16_t *)a.out + t * a.ldo + c) = o;
  }
}

template <bool VEC>
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a) {
  constexpr int C = VEC ? 8 : 1;
  const uint32_t per = (uint32_t)(a.N / C);
  // (a dispatch holds fewer threads than the largest results have elements)
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.T * per;
       i += (int64_t)gridDim.x * kThreads) {
    const int64_t t = i / per;
    combine<VEC>(a, t, C * (i - t * per));
  }
}

}  // namespace

hipError_t launch_expert_plan(const PlanArgs &a, hipStream_t s) {
  // A run of its own for every thousand pairs, beyond two thousand: a run's rounds take
  // 2 us each (4000 pairs of 32 experts in one run 10.2 us, in four 4.8 and 2.2 to count).
  const int64_t parts = std::min<int64_t>((a.pairs + kPlanThreads - 1) / kPlanThreads, kPlanParts);
  const dim3 grid((unsigned)(parts <= 2 ? 1 : parts));
  if (grid.x > 1) hipLaunchKernelGGL(plan_count_kernel, grid, dim3(kPlanThreads), 0, s, a);
  hipLaunchKernelGGL(plan_place_kernel, grid, dim3(kPlanThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_route(const RouteArgs &a, const PlanArgs &p, hipStream_t s) {
  if (a.T == 0) return launch_expert_plan(p, s);
  const bool few = a.T <= 2 * kPlanWaves && p.pairs <= kFewPairs;
  const dim3 grid((unsigned)((a.T + kThreads / 64 - 1) / (kThreads / 64))), block(kThreads);
  auto with = [&](auto ne, auto bias) {
    constexpr int NE = decltype(ne)::value;
    constexpr bool B = decltype(bias)::value;
    if (few)
      hipLaunchKernelGGL((route_few_kernel<NE, B>), dim3(1), dim3(kPlanThreads), 0, s, a, p);
    else
      hipLaunchKernelGGL((route_kernel<NE, B>), grid, block, 0, s, a);
  };
  auto go = [&](auto ne) {
    if (a.bias) with(ne, std::true_type{});
    else with(ne, std::false_type{});
  };
  if (a.E <= 64) go(std::integral_constant<int, 1>{});
  else if (a.E <= 128) go(std::integral_constant<int, 2>{});
  else if (a.E <= 256) go(std::integral_constant<int, 4>{});
  else if (a.E <= 512) go(std::integral_constant<int, 8>{});
  else go(std::integral_constant<int, 16>{});
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || few ? e : launch_expert_plan(p, s);
}

hipError_t launch_combine(const CombineArgs &a, hipStream_t s) {
  const int64_t yb = a.y_f32 ? 4 : 2, ob = a.out_f32 ? 4 : 2;
  const bool vec =
      a.N % 8 == 0 && ((a.ldy * yb | a.ldo * ob | (a.residual ? a.ldr * 2 : 0)) & 15) == 0 &&
      (((uintptr_t)a.y | (uintptr_t)a.out | (uintptr_t)a.residual) & 15) == 0;
  const int64_t n = std::min<int64_t>((a.T * (a.N / (vec ? 8 : 1)) + kThreads - 1) / kThreads, 1 << 22);
  if (vec) hipLaunchKernelGGL(combine_kernel<true>, dim3((unsigned)n), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(combine_kernel<false>, dim3((unsigned)n), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace mxq
