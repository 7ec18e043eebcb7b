// attn_paged_device.h -- what the two kernels of attention over the paged cache
// share: softmax weights, packed blocks to bf16, the batch and its partial results.
#pragma once

#include "mxq_device.h"
#include "mxq_internal.h"

namespace mxq {

namespace {

typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef unsigned short us8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s4 lds_s4;

constexpr int kD = 128;
constexpr int kRowBytes = 2 * kD;        // of a token's dequantized values in LDS
constexpr int kFewChunk = 32;            // tokens of a step of the kernel for few rows
constexpr float kLog2e = 1.44269504f;

// Softmax weights: e^d in float32 for float32 results (2^t with t = d log2 e, and
// what t lost in rounding as a first-order factor, kept finite for d = -inf; a NaN
// stays), 2^d of scores that carry the factor log2 e for bf16 ones.
template <bool F32>
__device__ inline float weight(float d) {
  if constexpr (!F32) return __builtin_amdgcn_exp2f(d);
  const float t = d * kLog2e;
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, __builtin_amdgcn_fmed3f(fmaf(t, -0.693147181f, d), -1.f, 1.f), e);
}
template <bool F32>
constexpr float kUnit = F32 ? 1.f : kLog2e;
// The softmax reference is raised (and O rescaled) only when a score passes it by
// more than this: the probabilities are then up to e^4.
template <bool F32>
constexpr float kSlack = 4.f * kUnit<F32>;

// The value of lane ^ 32.
__device__ inline float other_half(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// ---------------------------------------------------------------------------
// Packed blocks to bf16.

struct RawBlock {
  uint32_t w[8];                         // 4 m bytes
};

template <int M>
__device__ __forceinline__ void load_block(const uint8_t *p, RawBlock &r) {
  if constexpr (M == 4 || M == 8) {
#pragma unroll
    for (int i = 0; i < M / 4; ++i) {
      const u4 a = *(const u4 *)(p + 16 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) r.w[4 * i + k] = a[k];
    }
  } else if constexpr (M == 6) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const u2 a = *(const u2 *)(p + 8 * i);
      r.w[2 * i] = a[0];
      r.w[2 * i + 1] = a[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) r.w[i] = *(const uint32_t *)(p + 4 * i);
  }
}

// Slot i of eight values holds element slot_elem(m, i): 4- and 6-bit blocks yield
// the even elements, then the odd ones.
__device__ constexpr bool split_slots(int m) { return m == 4 || m == 6; }

// (a & m) | (b & ~m) for m = 0x0F0F0F0F; the mask is opaque to the compiler, which
// would split a constant one into two instructions.
__device__ inline uint32_t low_nibbles_else(uint32_t a, uint32_t b) {
  uint32_t m;
  asm("s_mov_b32 %0, 0x0f0f0f0f" : "=s"(m));
  return (a & m) | (b & ~m);
}

// The largest exponent whose scale keeps the arithmetic below inside the float
// range; a block beyond it is dequantized there and scaled again.
constexpr int max_exp(int m) { return m == 4 ? 247 : 253; }

// Group j (eight values) of a block, in slot order: q * 2^(E - 127 - (m - 2)), in two
// parts (so that a caller can put other work between them): integers, four values each.
struct Ints {
  uint32_t b0, b1;
};
template <int M>
__device__ __forceinline__ Ints ints8(const RawBlock &r, int j) {
  Ints y;
  if constexpr (M == 4) {
    // two's complement nibbles -> bytes of sign and magnitude 0..8, whose FP8
    // (e4m3) value is linear, k 2^-9
    const uint32_t w = r.w[j];
    const uint32_t sg = w & 0x88888888u, one = sg >> 3;
    const uint32_t mag = (w ^ ((one << 4) - one)) + one;
    y.b0 = low_nibbles_else(mag, sg << 4);
    y.b1 = low_nibbles_else(mag >> 4, sg);
  } else if constexpr (M == 8) {
    y.b0 = r.w[2 * j] ^ 0x80808080u;                       // bytes u = q + 128
    y.b1 = r.w[2 * j + 1] ^ 0x80808080u;
  } else if constexpr (M == 6) {
    // bytes u = q + 32; byte i of the top word: bits 7:6 and 5:4 (3:2 and 1:0 in
    // the odd groups) are the top bits of elements 2i and 2i + 1
    const uint32_t w = r.w[j], tw = r.w[4 + (j >> 1)] << (4 * (j & 1));
    y.b0 = low_nibbles_else(w, (tw >> 2) & 0x30303030u) ^ 0x20202020u;
    y.b1 = low_nibbles_else(w >> 4, tw & 0x30303030u) ^ 0x20202020u;
  } else {
    const int b = 24 * j, lo = b >> 5, sh = b & 31;
    uint32_t w = r.w[lo] >> sh;
    if (sh > 8) w |= r.w[lo + 1] << (32 - sh);
    y.b0 = w;                                              // eight 3-bit fields
    y.b1 = w >> 12;
  }
  return y;
}
// The factor that four() takes, of a block with exponent E.
template <int M>
__device__ __forceinline__ float factor(int E) {
  if constexpr (M == 4) return __uint_as_float((uint32_t)(min(E, max_exp(4)) + 7) << 23);
  return __builtin_amdgcn_ldexpf(1.f, min(E, max_exp(M)) - 127 - (M - 2));
}
// Four values from one of the two integers.
template <int M>
__device__ __forceinline__ bf4 four(uint32_t u, float sc) {
  if constexpr (M == 4) {                                  // the conversion applies the scale
    const bf2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, sc, false);
    const bf2 y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, sc, true);
    return bf4{x[0], x[1], y[0], y[1]};
  } else {
    float x[4];
    if constexpr (M == 3) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (float)(int)__builtin_amdgcn_sbfe((int)u, 3 * i, 3) * sc;
    } else {
      // u sc - 2^(M - 1) sc is exact, in one rounding
      const float off = sc * -(float)(1 << (M - 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = fmaf((float)((u >> (8 * i)) & 255u), sc, off);
    }
    return bf4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
  }
}
__device__ __forceinline__ bf8 both(bf4 x, bf4 y) {
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int M>
__device__ __forceinline__ bf8 dequant8(const RawBlock &r, int j, int E) {
  const Ints u = ints8<M>(r, j);
  const float sc = factor<M>(E);
  return both(four<M>(u.b0, sc), four<M>(u.b1, sc));
}

// The rest of the scale of blocks beyond max_exp.  (E = 255 is no exception: the
// quantizer writes zero mantissas with it.)  -2^128, the full clamp's lowest mantissa
// with E = 254, counts as bf16's lowest value: as an infinity it would be a NaN in the
// rows that do not see its token, times their probability of zero.  (As bits it is the one
// above the lowest value; a float maximum spills registers in the kernel for few rows.)
template <int M>
__device__ __forceinline__ void big_scale(bf8 &v, int E) {
  const float f = __builtin_amdgcn_ldexpf(1.f, max(E - max_exp(M), 0));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)((float)v[i] * f);
  const us8 low = {0xFF7F, 0xFF7F, 0xFF7F, 0xFF7F, 0xFF7F, 0xFF7F, 0xFF7F, 0xFF7F};
  v = __builtin_bit_cast(bf8, __builtin_elementwise_min(__builtin_bit_cast(us8, v), low));
}

// ---------------------------------------------------------------------------
// The batch.

// v[i], without an indexed array (which would go to scratch memory).
__device__ inline int pick(const int (&v)[4], int i) {
  return i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : v[3];
}

// A sequence's rows and tokens, as the kernel may use them.
struct Seq {
  int s, row0, n;                        // its first query row, and how many are computed
  int p0;                                // that row's position: the rows of q are the last tokens
  int len;                               // cached tokens
  int pre;                               // the tokens that every row sees
};
__device__ inline Seq seq_of(const AttnPagedArgs &a, int s, int begin, int end, int kv_len, int prefix) {
  Seq q;
  q.s = s;
  const int T = (int)a.T;
  const int c0 = min(max(begin, 0), T), c1 = min(max(end, c0), T);
  q.row0 = c0;
  q.n = min(c1 - c0, (int)a.max_q);
  int64_t len = min((int64_t)kv_len, a.max_kv);
  len = min(len, a.table_pages << a.geo.lg_page);
  q.len = (int)max(len, (int64_t)0);
  q.p0 = q.len - (c1 - c0);
  q.pre = min(max(prefix, 0), q.len);
  return q;
}
__device__ inline Seq seq_at(const AttnPagedArgs &a, int s) {
  return seq_of(a, s, a.cu_q[s], a.cu_q[s + 1], a.kv_len[s], a.prefix ? a.prefix[s] : 0);
}

// The steps (of TOK tokens) that rows at positions p_lo .. p_hi need: those of the
// prefix, then those from the first window on.
struct Steps {
  int pre, shift, count;                 // step v < pre is v, another v + shift
};
template <int TOK>
__device__ inline Steps steps_of(const AttnPagedArgs &a, const Seq &q, int64_t p_lo, int64_t p_hi) {
  Steps st;
  const int hi = (int)((min((int64_t)q.len, max(p_hi + 1, (int64_t)0)) + TOK - 1) / TOK);
  const int lo = a.window ? (int)(max(p_lo - a.window + 1, (int64_t)0) / TOK) : 0;
  st.pre = (q.pre + TOK - 1) / TOK;
  if (st.pre >= lo) {
    st.count = max(hi, st.pre);
    st.pre = st.shift = 0;
  } else {
    st.shift = lo - st.pre;
    st.count = st.pre + max(hi - lo, 0);
  }
  return st;
}

// Partial results of the splits: (maximum, sum) [parts][T Hq], padded to 16 bytes, then
// the unscaled outputs [parts][T Hq][128], `parts` being the larger number of splits of
// the two kernels.
__device__ inline float *part_ml(const AttnPagedArgs &a, int split, int64_t row) {
  return a.work + (split * a.T * a.Hq + row) * 2;
}
__device__ inline float *part_o(const AttnPagedArgs &a, int split, int64_t row) {
  return a.work + (a.parts * a.T * a.Hq + 1) / 2 * 4 + (split * a.T * a.Hq + row) * kD;
}

// The N scores x, capped: cap tanh(x sc / cap), in the unit of the softmax.
template <bool F32, int N, class V>
__device__ __forceinline__ void cap_scores(V &x, float sc, float cap, float k, float two) {
  // tanh y = 1 - 2 / (e^2y + 1) is good to 2.6 x 2^-23 of 1, so the score to that part of
  // the cap: 2e-5 at 64, a hundredth of what rounding its weight to bf16 costs.  Larger caps
  // take the series below 1/8 (its next term is 2^-29 of it), so that the error is a part
  // of the score.  (2048 tokens over 8192, 64 query and 8 KV heads: 690 us and 778.)
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = cap * tanhf(x[i] * sc / cap);
  } else if (cap <= 64.f) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = __builtin_amdgcn_exp2f(x[i] * sc * k);
      x[i] = fmaf(two, __builtin_amdgcn_rcpf(e + 1.f), cap) * kUnit<F32>;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = x[i] * sc, t = z * k, u = t * t;   // y = t s, s = ln 2 / 2
      constexpr float s2 = 0.120113253f;
      const float e = __builtin_amdgcn_exp2f(t);
      const float p = fmaf(u, fmaf(u, fmaf(u, -17.f / 315.f * s2 * s2 * s2, 2.f / 15.f * s2 * s2), s2 / -3.f), 1.f);
      x[i] = (fabsf(t) < 0.36f ? z * p : cap * fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f)) * kUnit<F32>;
    }
  }
}

}  // namespace
}  // namespace mxq
