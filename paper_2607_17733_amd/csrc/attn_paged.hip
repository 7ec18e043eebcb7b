// attn_paged.hip -- attention of new tokens over the paged MXINT KV cache
// (include/mxq.h states the operation).
//
// A sequence's n new tokens and the G query heads of a KV head make n G query
// rows that share K and V (row r: token r / G, head r % G).  A workgroup takes a
// tile of them and walks the cached tokens, 64 at a time, with a running maximum
// and sum of the softmax (one pass over K and V):
//   S^T = K Q^T     32x32x16 bf16 products, a lane holding one query row's scores
//                   of 32 of the 64 tokens (its partner, lane ^ 32, the others);
//   O^T += V^T P^T  takes the same lane's probabilities as they come out of the
//                   softmax: the order of the tokens over the reduction is free,
//                   and V follows it.
// So the statistics and the rescaling of O are a lane's own, and P never leaves
// the registers.  K and V are dequantized once per workgroup into LDS as bf16,
// which is exact (at most 8 significant bits): a wave per 32-value block of the
// row, a lane per token, so that widths are uniform over a wave.
//
// Sequences with at most 16 query rows per KV head (decoding, drafted tokens) have
// a kernel of their own: bytes and dequantization bound them, not products.  There
// each wave takes chunks of 32 tokens by itself, without a barrier, dequantizes K
// straight into the operand of 16x16x32 products and V into its own LDS rows, and
// the waves are merged at the end.  The tokens of a sequence are split over
// workgroups where there are few rows; the splits' results are merged in order.
#include <algorithm>

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
typedef __attribute__((address_space(3))) s4 lds_s4;

constexpr int kD = 128;
constexpr int kTok = 64;                 // tokens per step
constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;       // query rows of a tile
constexpr int kFewRows = 16;             // query rows of the kernel for few
constexpr int kMaxSplits = 256;
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
__device__ __forceinline__ void load_block(const uint8_t *p, int m, RawBlock &r) {
  if (m == 4) load_block<4>(p, r);
  else if (m == 8) load_block<8>(p, r);
  else if (m == 6) load_block<6>(p, r);
  else load_block<3>(p, r);
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
constexpr int max_exp(int m) { return m == 3 ? 255 : m == 4 ? 247 : 253; }

// Group j (eight values) of a block, in slot order: q * 2^(E - 127 - (m - 2)).
template <int M>
__device__ __forceinline__ bf8 dequant8(const RawBlock &r, int j, int E) {
  if constexpr (M == 4) {
    // two's complement nibbles -> bytes of sign and magnitude 0..8, whose FP8
    // (e4m3) value is linear, k 2^-9; the conversion applies the block's scale
    const uint32_t w = r.w[j];
    const uint32_t sg = w & 0x88888888u, one = sg >> 3;
    const uint32_t mag = (w ^ ((one << 4) - one)) + one;
    const uint32_t ev = low_nibbles_else(mag, sg << 4), od = low_nibbles_else(mag >> 4, sg);
    const float sc = __uint_as_float((uint32_t)(min(E, max_exp(4)) + 7) << 23);
    bf2 v[4];
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(ev, sc, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(ev, sc, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(od, sc, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(od, sc, true);
    return bf8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
  } else {
    const float sc = __builtin_amdgcn_ldexpf(1.f, min(E, max_exp(M)) - 127 - (M - 2));
    float x[8];
    if constexpr (M == 3) {
      const int b = 24 * j, lo = b >> 5, sh = b & 31;
      uint32_t w = r.w[lo] >> sh;
      if (sh > 8) w |= r.w[lo + 1] << (32 - sh);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (float)(int)__builtin_amdgcn_sbfe((int)w, 3 * i, 3) * sc;
    } else {
      // bytes u = q + 2^(M - 1); u sc - 2^(M - 1) sc is exact, in one rounding
      uint32_t b0, b1;
      if constexpr (M == 8) {
        b0 = r.w[2 * j] ^ 0x80808080u;
        b1 = r.w[2 * j + 1] ^ 0x80808080u;
      } else {
        // byte i of the top word: bits 7:6 and 5:4 (3:2 and 1:0 in the odd groups)
        // are the top bits of elements 2i and 2i + 1
        const uint32_t w = r.w[j], tw = r.w[4 + (j >> 1)] << (4 * (j & 1));
        b0 = low_nibbles_else(w, (tw >> 2) & 0x30303030u) ^ 0x20202020u;
        b1 = low_nibbles_else(w >> 4, tw & 0x30303030u) ^ 0x20202020u;
      }
      const float off = sc * -(float)(1 << (M - 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = fmaf((float)((b0 >> (8 * i)) & 255u), sc, off);
        x[4 + i] = fmaf((float)((b1 >> (8 * i)) & 255u), sc, off);
      }
    }
    bf8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)x[i];
    return y;
  }
}

// LDS rows of a token's 128 bf16 values: sixteen chunks of 16 bytes, chunk c of
// token t at c ^ swizzle(t).  Sixteen tokens' writes or operand reads of one chunk
// and a transposing read (four tokens, four adjacent chunks) lie in distinct banks.
constexpr int kRowBytes = 2 * kD;
constexpr int kTileBytes = kTok * kRowBytes;
__device__ inline int swizzle(int t) { return 4 * (t & 3) + ((t >> 2) & 3); }

// The rest of the scale of blocks beyond max_exp.  (E = 255 is no exception: the
// quantizer writes zero mantissas with it.)
template <int M>
__device__ __forceinline__ void big_scale(bf8 &v, int E) {
  if constexpr (M == 3) return;
  const float f = __builtin_amdgcn_ldexpf(1.f, max(E - max_exp(M), 0));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)((float)v[i] * f);
}

// A token's block b to its LDS row.
template <int M>
__device__ __forceinline__ void store_block(const RawBlock &r, int E, uint8_t *tile, int t, int b) {
  bf8 v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = dequant8<M>(r, j, E);
  if (__any(E > max_exp(M))) {
#pragma unroll
    for (int j = 0; j < 4; ++j) big_scale<M>(v[j], E);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *(bf8 *)(tile + t * kRowBytes + 16 * ((4 * b + j) ^ swizzle(t))) = v[j];
}
__device__ __forceinline__ void store_block(const RawBlock &r, int m, int E, uint8_t *tile, int t, int b) {
  if (m == 4) store_block<4>(r, E, tile, t, b);
  else if (m == 8) store_block<8>(r, E, tile, t, b);
  else if (m == 6) store_block<6>(r, E, tile, t, b);
  else store_block<3>(r, E, tile, t, b);
}

// ---------------------------------------------------------------------------
// The batch.

// v[i], without an indexed array (which would go to scratch memory).
__device__ inline int pick(const int (&v)[4], int i) {
  return i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : v[3];
}

// A sequence's rows and tokens, as the kernel may use them.
struct Seq {
  int s, row0, n;                        // its first query row, and how many
  int len;                               // cached tokens
  int pre;                               // the tokens that every row sees
};
__device__ inline Seq seq_at(const AttnPagedArgs &a, int s) {
  Seq q;
  q.s = s;
  const int T = (int)a.T;
  const int c0 = min(max(a.cu_q[s], 0), T), c1 = min(max(a.cu_q[s + 1], c0), T);
  q.row0 = c0;
  q.n = c1 - c0;
  int64_t len = min((int64_t)a.kv_len[s], a.max_kv);
  len = min(len, a.table_pages << a.geo.lg_page);
  q.len = (int)max(len, (int64_t)0);
  q.pre = a.prefix ? min(max(a.prefix[s], 0), q.len) : 0;
  return q;
}

// The tiles of `rows` query rows of all sequences are numbered with gaps: those of
// sequence s begin at floor(cu_q[s] G / rows) + s.  No two sequences meet (a
// sequence of n rows has at most floor(end / rows) - floor(begin / rows) + 1
// tiles), and floor(T G / rows) + S numbers are enough, so that the launch needs
// no look at the device's lengths.  The sequence of a number, by 64-way search
// (-1: a gap).
__device__ inline int find_seq(const AttnPagedArgs &a, int64_t number, int rows, int &tile) {
  const int lane = threadIdx.x & 63;
  auto start = [&](int s) { return (int64_t)max(a.cu_q[s], 0) * a.G / rows + s; };
  int lo = 0, cnt = (int)a.S;
  for (;;) {
    const int step = (cnt + 63) / 64, s = lo + lane * step;
    const bool le = s < lo + cnt && start(s) <= number;
    const int k = __popcll(__ballot(le));
    if (k == 0) return -1;
    lo += (k - 1) * step;
    if (step == 1) break;
    cnt = min(step, (int)a.S - lo);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  tile = (int)(number - start(lo));
  return lo;
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

// Partial results of the splits: (maximum, sum) [parts][T Hq], then the unscaled
// outputs [parts][T Hq][128], `parts` being the larger number of splits of the two
// kernels.
__device__ inline float *part_ml(const AttnPagedArgs &a, int split, int64_t row) {
  return a.work + (split * a.T * a.Hq + row) * 2;
}
__device__ inline float *part_o(const AttnPagedArgs &a, int split, int64_t row) {
  return a.work + a.parts * a.T * a.Hq * 2 + (split * a.T * a.Hq + row) * kD;
}

template <bool F32>
__device__ inline float capped(float x, float cap) {
  if constexpr (F32) return cap * tanhf(x / cap);
  // tanh y = 1 - 2 / (e^2y + 1), its error 2^-23 of 1
  const float e = __builtin_amdgcn_exp2f(x * (2.f * kLog2e / cap));
  return fmaf(-2.f * cap, __builtin_amdgcn_rcpf(e + 1.f), cap);
}

template <bool F32>
__global__ __launch_bounds__(64 * kWaves, 2)
void attn_tile_kernel(AttnPagedArgs a, int splits, int64_t numbers, int few) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][2][kTileBytes];   // [buffer][K, V]
  const PageGeo &g = a.geo;
  const int t = threadIdx.x, lane = t & 63, h = lane >> 5, x = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  // KV heads run fastest, so that with eight of them an XCD reads one head's
  // pages; a sequence's last tiles, which see most tokens, come first
  const int Hkv = (int)g.Hkv, G = a.G;
  const uint32_t rest = blockIdx.x / (uint32_t)Hkv;
  const int kvh = (int)(blockIdx.x - rest * (uint32_t)Hkv);
  const int64_t number = numbers - 1 - rest / (uint32_t)splits;
  const int split = (int)(rest % (uint32_t)splits);
  int tile;
  const int s = find_seq(a, number, kRows, tile);
  if (s < 0) return;
  const Seq q = seq_at(a, s);
  const int64_t rows = (int64_t)q.n * G, r0 = (int64_t)tile * kRows;
  if (r0 >= rows || (few && rows <= kFewRows)) return;
  const int64_t p0 = (int64_t)q.len - q.n;                 // the first row's position
  const Steps st = steps_of<kTok>(a, q, p0 + r0 / G, p0 + (min(r0 + kRows, rows) - 1) / G);
  const int v0 = (int)((int64_t)st.count * split / splits);
  const int v1 = (int)((int64_t)st.count * (split + 1) / splits);

  // this lane's query row, and the wave's first and last position
  const int64_t wr = r0 + 32 * wave;
  const bool live = wr < rows;                             // of the wave
  const int64_t r = min(wr + x, rows - 1);
  const int tok = (int)(r / G), hd = kvh * G + (int)(r - (int64_t)tok * G);
  const int p = (int)(p0 + tok);
  const int pw0 = (int)(p0 + min(wr, rows - 1) / G), pw1 = (int)(p0 + (min(wr + 32, rows) - 1) / G);
  const int window = (int)(a.window && a.window < INT32_MAX ? a.window : INT32_MAX);

  // The score product's Q operand: 16 values of the reduction per product, lane
  // half h taking eight, in the slot order of their block.  A negative scale goes
  // into its sign; for a scale of zero Q is zero (a masked score, -inf, is scaled).
  bf8 qop[8];
  {
    const uint16_t *src = a.q + (int64_t)(q.row0 + tok) * a.q_ts + hd * a.q_hs;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      u4 w = *(const u4 *)(src + 16 * ks + 8 * h);
      w = a.scale == 0.f ? u4{0u, 0u, 0u, 0u} : w ^ u4{sign, sign, sign, sign};
      if (split_slots(g.m[ks >> 1]))
        w = u4{__builtin_amdgcn_perm(w[1], w[0], 0x05040100), __builtin_amdgcn_perm(w[3], w[2], 0x05040100),
               __builtin_amdgcn_perm(w[1], w[0], 0x07060302), __builtin_amdgcn_perm(w[3], w[2], 0x07060302)};
      qop[ks] = __builtin_bit_cast(bf8, w);
    }
  }
  const float sc = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * (a.softcap > 0.f ? 1.f : kUnit<F32>);
  const float slope = a.slopes ? a.slopes[hd] * kUnit<F32> : 0.f;

  const float ninf = -__builtin_inff();
  float m = ninf, ref = 0.f, l = 0.f;                      // l: this lane's tokens
  f16v o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

  // Dequantization: this wave's block, this lane's token of a step.  Tokens past
  // the last are the last one (weight 0).
  const int blk = wave, bm = pick(g.m, blk);
  const int64_t plane = (int64_t)pick(g.off, blk) << g.lg_page;
  const int page_mask = (1 << g.lg_page) - 1;
  const int32_t *pages = a.table + (int64_t)s * a.ld_table;
  RawBlock rk, rv;
  uint32_t ek, ev;
  auto token_of = [&](int v) { return min((v < st.pre ? v : v + st.shift) * kTok + lane, q.len - 1); };
  auto page_of = [&](int v) { return pages[token_of(min(v, v1 - 1)) >> g.lg_page]; };
  auto fetch = [&](int v, int page) __attribute__((always_inline)) {
    const bool hole = page < 0 || page >= g.pages;
    const int i = token_of(v) & page_mask;
    const int64_t run = ((int64_t)(hole ? 0 : page) * Hkv + kvh) << g.lg_page;
    const int64_t at = run * g.row + plane + i * 4 * bm;
    load_block(a.k_mant + at, bm, rk);
    load_block(a.v_mant + at, bm, rv);
    ek = a.k_exp[(run + i) * 4 + blk];
    ev = a.v_exp[(run + i) * 4 + blk];
    if (hole) {                                            // zero rows
#pragma unroll
      for (int k = 0; k < 8; ++k) rk.w[k] = rv.w[k] = 0u;
    }
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
    store_block(rk, bm, (int)ek, lds[buf][0], lane, blk);
    store_block(rv, bm, (int)ev, lds[buf][1], lane, blk);
  };

  if (v0 < v1) {
    const int page = page_of(v0);
    int next = page_of(v0 + 1);
    fetch(v0, page);
    put(0);
    for (int v = v0; v < v1; ++v) {
      const int buf = (v - v0) & 1;
      __syncthreads();                                     // this step's rows are there, the last one's read
      if (v + 1 < v1) {
        fetch(v + 1, next);
        next = page_of(v + 2);
      }
      const int t0 = (v < st.pre ? v : v + st.shift) * kTok;
      if (live && ((t0 <= pw1 && pw0 - t0 - kTok + 1 < window) || t0 < q.pre)) {
        // scores
        f16v sa[2];
        const uint8_t *kt = lds[buf][0] + x * kRowBytes;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int i = 0; i < 16; ++i) sa[u][i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            const bf8 k = *(const bf8 *)(kt + u * 32 * kRowBytes + 16 * ((2 * ks + h) ^ swizzle(x)));
            sa[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qop[ks], sa[u], 0, 0, 0);
          }
        }
        // value i of half u is token t0 + 4 h + c(u, i)
        auto c = [](int u, int i) { return 32 * u + 8 * (i >> 2) + (i & 3); };
        float scale = sc;
        if (a.softcap > 0.f || a.slopes) {
          const float rel = (float)(p - t0 - 4 * h);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float y = sa[u][i] * sc;
              if (a.softcap > 0.f) y = capped<F32>(y, a.softcap) * kUnit<F32>;
              sa[u][i] = fmaf(-slope, fabsf(rel - (float)c(u, i)), y);
            }
          scale = 1.f;
        }
        // masks, for steps that not every row of the wave sees whole
        if (t0 + kTok - 1 > pw0 || pw1 - t0 >= window || t0 + kTok > q.len) {
          const int rel = p - t0 - 4 * h, pre = q.pre - t0 - 4 * h, end = q.len - t0 - 4 * h;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int k = c(u, i);
              const bool see = ((k <= rel && rel - k < window) || k < pre) && k < end;
              if (!see) sa[u][i] = ninf;
            }
        }
        float top = sa[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, sa[u][i]);
        top = fmaxf(top, other_half(top));
        top = top == ninf ? ninf : top * scale;
        if (__any(top > m + kSlack<F32> || (m == ninf && top != ninf))) {
          const float nm = fmaxf(m, top);
          const float alpha = m == ninf ? 0.f : weight<F32>(m - nm);
          m = nm;
          ref = nm == ninf ? 0.f : nm;                     // scores of -inf weigh 0
          l *= alpha;
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            sa[u][i] = weight<F32>(fmaf(sa[u][i], scale, -ref));
            l += sa[u][i];
          }
        // values: product z takes tokens 16 z ..; lane half h holds its tokens
        // 4 h .. 4 h + 3 and 8 + 4 h ..
        const int n = lane & 15, w4 = lane >> 4 & 1;
        const uint8_t *vt = lds[buf][1] + (4 * h + (n >> 2)) * kRowBytes + 8 * (n & 1);
        const int col = 2 * w4 + ((n & 3) >> 1);
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          float e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = sa[z >> 1][8 * (z & 1) + i];
          constexpr int kTerms = F32 ? 3 : 1;
          bf8 pt[kTerms];
#pragma unroll
          for (int k = 0; k < kTerms; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              pt[k][i] = (__bf16)e[i];
              if constexpr (F32) e[i] -= (float)pt[k][i];
            }
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) {
            const uint8_t *v0p = vt + 16 * z * kRowBytes + 16 * ((4 * dt + col) ^ (4 * (n >> 2) + h));
            const uint8_t *v1p = vt + (16 * z + 8) * kRowBytes + 16 * ((4 * dt + col) ^ (4 * (n >> 2) + h + 2));
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)v0p);
            const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)v1p);
            const bf8 vv = __builtin_bit_cast(bf8, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int k = 0; k < kTerms; ++k)
              o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, pt[k], o[dt], 0, 0, 0);
          }
        }
      }
      if (v + 1 < v1) put(buf ^ 1);
    }
  }
  if (wr + x >= rows) return;
  l += other_half(l);
  const int64_t row = (int64_t)(q.row0 + tok) * a.Hq + hd;
  const bool whole = splits == 1;
  const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
  if (!whole) {
    if (h == 0) *(f2 *)part_ml(a, split, row) = f2{m, l};
    if (v0 >= v1) return;
  }
  float *of = whole ? (float *)a.o + row * kD : part_o(a, split, row);
  uint16_t *ob = (uint16_t *)a.o + row * kD;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // slots 4 h .. 4 h + 3 of eight values; split slots hold the even (h = 0) and
      // odd (h = 1) elements: the partners exchange two
      f4 y = {o[dt][4 * k] * inv, o[dt][4 * k + 1] * inv, o[dt][4 * k + 2] * inv, o[dt][4 * k + 3] * inv};
      if (split_slots(g.m[dt])) {
        const auto e = __builtin_amdgcn_permlane32_swap(__float_as_uint(y[0]), __float_as_uint(y[2]), false, false);
        const auto f = __builtin_amdgcn_permlane32_swap(__float_as_uint(y[1]), __float_as_uint(y[3]), false, false);
        y = f4{__uint_as_float(e[0]), __uint_as_float(e[1]), __uint_as_float(f[0]), __uint_as_float(f[1])};
      }
      const int d = 32 * dt + 8 * k + 4 * h;
      if (!whole || F32) *(f4 *)(of + d) = y;
      else *(bf4 *)(ob + d) = bf4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
    }
}

// ---------------------------------------------------------------------------
// Few rows.

constexpr int kChunk = 32;               // tokens of a wave's step
constexpr int kFewWaves = 4;
// LDS rows of a wave's 32 dequantized V tokens: chunk c (16 bytes) of token t at c ^
// swizzle: eight tokens' writes of one chunk, and a transposing read's eight tokens
// of two adjacent chunks, lie in distinct banks.
constexpr int kFewBytes = kChunk * kRowBytes;
__device__ inline int few_swizzle(int t) { return 2 * (t & 7) + ((t >> 3) & 1); }

// The widths of a row's blocks: N3 3-bit, N4 4-bit, N6 6-bit and N8 8-bit blocks, in
// that order.  Rows of one width are read a block per lane (lane group g: block g,
// product j: its group j), others a group of each block (product j: block j, lane
// group g: its group g), so that all lanes run one width's code.
template <int N3, int N4, int N6, int N8>
struct Mix {
  static constexpr bool kUniform = N3 == 4 || N4 == 4 || N6 == 4 || N8 == 4;
  static constexpr int width(int b) {
    return b < N3 ? 3 : b < N3 + N4 ? 4 : b < N3 + N4 + N6 ? 6 : 8;
  }
  static constexpr int off(int b) { return b == 0 ? 0 : off(b - 1) + 4 * width(b - 1); }
  // words of product j that a lane loads, and where they begin
  static constexpr int words(int j) {
    return kUniform ? (j == 0 ? width(0) : 0) : width(j) == 4 ? 1 : 2;
  }
  static constexpr int start(int j) { return j == 0 ? 0 : start(j - 1) + words(j - 1); }
  static constexpr int kWords = start(4);
  // first value of the eight of (lane group g, product j)
  static constexpr __device__ int value(int g, int j) { return kUniform ? 32 * g + 8 * j : 32 * j + 8 * g; }
};

// A lane's share of a token's row: its packed words and the four exponents.
template <class Mx>
struct RawRow {
  uint32_t w[Mx::kWords];
  uint32_t ex;
};

// `plane` points at the page's first token, `i` is the token.
template <class Mx, int J>
__device__ __forceinline__ void load_group(const uint8_t *page, int lg_page, uint32_t i, int g,
                                           RawRow<Mx> &r) {
  constexpr int M = Mx::width(J), S = Mx::start(J);
  const uint8_t *p = page + (((uint32_t)Mx::off(J) << lg_page) + i * (4 * M));
  if constexpr (M == 4) {
    r.w[S] = *(const uint32_t *)(p + 4 * g);
  } else if constexpr (M == 6) {
    r.w[S] = *(const uint32_t *)(p + 4 * g);
    r.w[S + 1] = *(const uint32_t *)(p + 16 + 4 * (g >> 1));
  } else if constexpr (M == 8) {
    const u2 a = *(const u2 *)(p + 8 * g);
    r.w[S] = a[0];
    r.w[S + 1] = a[1];
  } else {                               // bytes 3 g .. 3 g + 2 of twelve
    const int at = (3 * g) & ~3;
    r.w[S] = *(const uint32_t *)(p + at);
    r.w[S + 1] = *(const uint32_t *)(p + (at < 8 ? at + 4 : 8));
  }
}
template <class Mx>
__device__ __forceinline__ void load_row(const uint8_t *page, int lg_page, uint32_t i, int g,
                                         RawRow<Mx> &r) {
  if constexpr (Mx::kUniform) {
    constexpr int M = Mx::width(0);
    RawBlock b;
    load_block<M>(page + ((((uint32_t)(4 * M * g)) << lg_page) + i * (4 * M)), b);
#pragma unroll
    for (int k = 0; k < M; ++k) r.w[k] = b.w[k];
  } else {
    load_group<Mx, 0>(page, lg_page, i, g, r);
    load_group<Mx, 1>(page, lg_page, i, g, r);
    load_group<Mx, 2>(page, lg_page, i, g, r);
    load_group<Mx, 3>(page, lg_page, i, g, r);
  }
}

// Product J's eight values, in slot order.
template <class Mx, int J>
__device__ __forceinline__ bf8 dequant_group(const RawRow<Mx> &r, int g) {
  constexpr int M = Mx::width(J), S = Mx::start(J);
  const int E = (int)__builtin_amdgcn_ubfe(r.ex, Mx::kUniform ? 8 * g : 8 * J, 8);
  RawBlock b;
  bf8 v;
  if constexpr (Mx::kUniform) {
#pragma unroll
    for (int k = 0; k < M; ++k) b.w[k] = r.w[k];
    v = dequant8<M>(b, J, E);
  } else {                               // as group 0 of a block
    if constexpr (M == 6) {
      b.w[0] = r.w[S];
      b.w[4] = r.w[S + 1] << (4 * (g & 1));
    } else if constexpr (M == 3) {
      b.w[0] = __builtin_amdgcn_alignbit(r.w[S + 1], r.w[S], 8 * ((3 * g) & 3));
    } else {
      b.w[0] = r.w[S];
      if constexpr (M == 8) b.w[1] = r.w[S + 1];
    }
    v = dequant8<M>(b, 0, E);
  }
  return v;
}
template <class Mx>
__device__ __forceinline__ void dequant_row(const RawRow<Mx> &r, int g, bool big, bf8 (&v)[4]) {
  v[0] = dequant_group<Mx, 0>(r, g);
  v[1] = dequant_group<Mx, 1>(r, g);
  v[2] = dequant_group<Mx, 2>(r, g);
  v[3] = dequant_group<Mx, 3>(r, g);
  if (big) {
    auto E = [&](int j) { return (int)__builtin_amdgcn_ubfe(r.ex, Mx::kUniform ? 8 * g : 8 * j, 8); };
    big_scale<Mx::width(0)>(v[0], E(0));
    big_scale<Mx::width(1)>(v[1], E(1));
    big_scale<Mx::width(2)>(v[2], E(2));
    big_scale<Mx::width(3)>(v[3], E(3));
  }
}

// Whether one of four exponents may pass max_exp.
__device__ inline bool has_big(uint32_t ex) {
  return (ex & (ex << 1) & (ex << 2) & 0x80808080u) != 0;
}

__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <bool F32, class Mx>
__global__ __launch_bounds__(64 * kFewWaves, 3)
void attn_few_kernel(AttnPagedArgs a, int splits) {
  __shared__ __attribute__((aligned(16))) uint8_t pool[kFewWaves][kFewBytes];
  __shared__ float mm[kFewWaves][kFewRows], ml[kFewWaves][kFewRows];
  const PageGeo &g = a.geo;
  const int t = threadIdx.x, lane = t & 63, gr = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint32_t Hkv = (uint32_t)g.Hkv;
  const int G = a.G;
  const uint32_t rest = blockIdx.x / Hkv;
  const int kvh = (int)(blockIdx.x - rest * Hkv);
  const int s = (int)(rest / (uint32_t)splits), split = (int)(rest - (uint32_t)s * (uint32_t)splits);
  const Seq q = seq_at(a, s);
  const int64_t rows = (int64_t)q.n * G;
  if (rows == 0 || rows > kFewRows) return;
  const int p0 = q.len - q.n;                              // the first row's position
  const Steps st = steps_of<kChunk>(a, q, p0, (int64_t)q.len - 1);
  const int v0 = (int)((int64_t)st.count * split / splits);
  const int v1 = (int)((int64_t)st.count * (split + 1) / splits);

  // this lane's query row (columns past the last repeat it)
  const int r = min(n, (int)rows - 1), tok = r / G, hd = kvh * G + r - tok * G, p = p0 + tok;
  const int window = (int)(a.window && a.window < INT32_MAX ? a.window : INT32_MAX);
  // product j of a score: the values of lane group gr, in slot order
  bf8 qop[4];
  {
    const uint16_t *src = a.q + (int64_t)(q.row0 + tok) * a.q_ts + hd * a.q_hs;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u4 w = *(const u4 *)(src + Mx::value(gr, j));
      w = a.scale == 0.f ? u4{0u, 0u, 0u, 0u} : w ^ u4{sign, sign, sign, sign};
      if (split_slots(Mx::width(j)))
        w = u4{__builtin_amdgcn_perm(w[1], w[0], 0x05040100), __builtin_amdgcn_perm(w[3], w[2], 0x05040100),
               __builtin_amdgcn_perm(w[1], w[0], 0x07060302), __builtin_amdgcn_perm(w[3], w[2], 0x07060302)};
      qop[j] = __builtin_bit_cast(bf8, w);
    }
  }
  const float sc = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * (a.softcap > 0.f ? 1.f : kUnit<F32>);
  const float slope = a.slopes ? a.slopes[hd] * kUnit<F32> : 0.f;
  const float ninf = -__builtin_inff();
  float m = ninf, ref = 0.f, l = 0.f;
  f4 o[8];                                                 // row n, slots 16 dt + 4 gr ..
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) o[dt] = f4{0.f, 0.f, 0.f, 0.f};

  // A chunk's halves of 16 tokens lie in one page each.  Tokens past the last are
  // the last one (weight 0), a half past the last the chunk's first.
  const int32_t *pages = a.table + (int64_t)s * a.ld_table;
  const int page_mask = (1 << g.lg_page) - 1, last = q.len - 1;
  RawRow<Mx> rk[2], rv[2];
  auto first_of = [&](int v) { return (v < st.pre ? v : v + st.shift) * kChunk; };
  auto fetch = [&](int v) __attribute__((always_inline)) {
    const int t0 = first_of(v);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int th = t0 + 16 * mt <= last ? t0 + 16 * mt : t0;
      const int page = pages[th >> g.lg_page];
      const bool hole = page < 0 || page >= g.pages;
      const int64_t run = ((int64_t)(hole ? 0 : page) * Hkv + kvh) << g.lg_page;
      const int i = min(th + n, last) & page_mask;
      const uint8_t *kp = a.k_mant + run * g.row, *vp = a.v_mant + run * g.row;
      load_row<Mx>(kp, g.lg_page, (uint32_t)i, gr, rk[mt]);
      load_row<Mx>(vp, g.lg_page, (uint32_t)i, gr, rv[mt]);
      rk[mt].ex = *(const uint32_t *)(a.k_exp + (run + i) * 4);
      rv[mt].ex = *(const uint32_t *)(a.v_exp + (run + i) * 4);
      if (hole) {                                          // zero rows
#pragma unroll
        for (int k = 0; k < Mx::kWords; ++k) rk[mt].w[k] = rv[mt].w[k] = 0u;
        rk[mt].ex = rv[mt].ex = 0u;
      }
    }
  };
  uint8_t *vs = pool[wave];
  if (v0 + wave < v1) fetch(v0 + wave);
  for (int v = v0 + wave; v < v1; v += kFewWaves) {
    const int t0 = first_of(v);
    const bool big = __any(has_big(rk[0].ex) || has_big(rk[1].ex) || has_big(rv[0].ex) || has_big(rv[1].ex));
    // scores: tokens 16 mt + 4 gr + i of row n
    f4 sa[2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      bf8 k[4];
      dequant_row(rk[mt], gr, big, k);
      sa[mt] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        sa[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], qop[j], sa[mt], 0, 0, 0);
    }
    wave_sync();                                           // the last chunk's V rows are consumed
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      bf8 w[4];
      dequant_row(rv[mt], gr, big, w);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(bf8 *)(vs + (16 * mt + n) * kRowBytes + 16 * ((Mx::value(gr, j) >> 3) ^ few_swizzle(n))) = w[j];
    }
    if (v + kFewWaves < v1) fetch(v + kFewWaves);
    wave_sync();
    float scale = sc;
    if (a.softcap > 0.f || a.slopes) {
      const float rel = (float)(p - t0 - 4 * gr);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = sa[mt][i] * sc;
          if (a.softcap > 0.f) y = capped<F32>(y, a.softcap) * kUnit<F32>;
          sa[mt][i] = fmaf(-slope, fabsf(rel - (float)(16 * mt + i)), y);
        }
      scale = 1.f;
    }
    if (t0 + kChunk - 1 > p0 || (q.len - 1) - t0 >= window || t0 + kChunk > q.len) {
      const int rel = p - t0 - 4 * gr, pre = q.pre - t0 - 4 * gr, end = q.len - t0 - 4 * gr;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 16 * mt + i;
          const bool see = ((k <= rel && rel - k < window) || k < pre) && k < end;
          if (!see) sa[mt][i] = ninf;
        }
    }
    float top = fmaxf(fmaxf(fmaxf(sa[0][0], sa[0][1]), fmaxf(sa[0][2], sa[0][3])),
                      fmaxf(fmaxf(sa[1][0], sa[1][1]), fmaxf(sa[1][2], sa[1][3])));
    top = top == ninf ? ninf : top * scale;
    if (__any(top > m + kSlack<F32> || (m == ninf && top != ninf))) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float nm = fmaxf(m, top);
      const float alpha = m == ninf ? 0.f : weight<F32>(m - nm);
      m = nm;
      ref = nm == ninf ? 0.f : nm;                         // scores of -inf weigh 0
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
    }
    float e[8];                                            // the product's slots: tokens 4 gr + i, 16 + 4 gr + i
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = weight<F32>(fmaf(sa[i >> 2][i & 3], scale, -ref));
      l += e[i];
    }
    constexpr int kTerms = F32 ? 3 : 1;
    bf8 pt[kTerms];
#pragma unroll
    for (int k = 0; k < kTerms; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pt[k][i] = (__bf16)e[i];
        if constexpr (F32) e[i] -= (float)pt[k][i];
      }
    const uint8_t *vp = vs + (4 * gr + (n >> 2)) * kRowBytes + 8 * (n & 1);
    const int sw = few_swizzle(4 * gr + (n >> 2)), col = (n & 3) >> 1;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const uint8_t *at = vp + 16 * ((2 * dt + col) ^ sw);
      const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)at);
      const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(at + 16 * kRowBytes));
      const bf8 vv = __builtin_bit_cast(bf8, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int k = 0; k < kTerms; ++k)
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[k], o[dt], 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // Merge the waves in order: each writes its outputs, weighted against the row's
  // largest reference, over its V rows.
  if (gr == 0) {
    mm[wave][n] = m;
    ml[wave][n] = l;
  }
  __syncthreads();
  float M = ninf;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) M = fmaxf(M, mm[w][n]);
  const float f = m == ninf ? 0.f : weight<F32>(m - M);
  float *mo = (float *)vs;                                 // [row][d]
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    const int d8 = 16 * dt + 8 * (gr >> 1);
    const bool sp = split_slots(Mx::width(dt >> 1));
#pragma unroll
    for (int i = 0; i < 4; ++i)                            // (0 without a finite score; a NaN stays)
      mo[n * kD + d8 + (sp ? 2 * i + (gr & 1) : 4 * (gr & 1) + i)] = o[dt][i] * f;
  }
  __syncthreads();
  for (int i = t; i < (int)rows * (kD / 4); i += 64 * kFewWaves) {
    const int row = i / (kD / 4), d = 4 * (i % (kD / 4));
    float M2 = ninf, L = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) M2 = fmaxf(M2, mm[w][row]);
    f4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      L += mm[w][row] == ninf ? ml[w][row] : ml[w][row] * weight<F32>(mm[w][row] - M2);
      O += *(const f4 *)((float *)pool[w] + row * kD + d);
    }
    const int tk = row / G;
    const int64_t at = (int64_t)(q.row0 + tk) * a.Hq + kvh * G + row - tk * G;
    if (splits > 1) {
      if (d == 0) *(f2 *)part_ml(a, split, at) = f2{M2, L};
      *(f4 *)(part_o(a, split, at) + d) = O;
    } else {
      O *= L == 0.f ? 0.f : 1.f / L;
      if (F32) *(f4 *)((float *)a.o + at * kD + d) = O;
      else *(bf4 *)((uint16_t *)a.o + at * kD + d) =
          bf4{(__bf16)O[0], (__bf16)O[1], (__bf16)O[2], (__bf16)O[3]};
    }
  }
}

// o[row] = the splits' partial results merged, in the order of the splits: half a
// wave per row.
template <bool F32>
__global__ __launch_bounds__(256) void attn_merge_kernel(AttnPagedArgs a, int tile, int few) {
  const int t = threadIdx.x, c = t & 31;
  const int64_t row = (int64_t)blockIdx.x * 8 + (t >> 5);
  if (row >= a.T * a.Hq) return;
  const int tok = (int)(row / a.Hq);
  if (tok < a.cu_q[0] || tok >= a.cu_q[a.S]) return;       // no sequence's row
  int splits = tile;
  if (tile != few) {                                       // which kernel had the row
    int lo = 0, hi = (int)a.S - 1;                         // the last sequence that begins at tok or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (a.cu_q[mid] <= tok) lo = mid;
      else hi = mid - 1;
    }
    if ((int64_t)(a.cu_q[lo + 1] - a.cu_q[lo]) * a.G <= kFewRows) splits = few;
    if (splits == 1) return;                               // written already
  }
  const float ninf = -__builtin_inff();
  float M = ninf;
  for (int s = c; s < splits; s += 32) M = fmaxf(M, part_ml(a, s, row)[0]);
#pragma unroll
  for (int w = 1; w < 32; w *= 2) M = fmaxf(M, __shfl_xor(M, w));
  const float ref = M == ninf ? 0.f : M;
  float L = 0.f;
  f4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const f2 ml = *(const f2 *)part_ml(a, s, row);
    // (a NaN sum has no maximum to go by, but counts)
    if (ml[0] == ninf && ml[1] == 0.f) continue;
    const float f = weight<F32>(ml[0] - ref);
    L += ml[1] * f;
    O += *(const f4 *)(part_o(a, s, row) + 4 * c) * f;
  }
  O *= L == 0.f ? 0.f : 1.f / L;
  if (F32) *(f4 *)((float *)a.o + row * kD + 4 * c) = O;
  else *(bf4 *)((uint16_t *)a.o + row * kD + 4 * c) =
      bf4{(__bf16)O[0], (__bf16)O[1], (__bf16)O[2], (__bf16)O[3]};
}

// The kernel for a row's widths, code = 125 n3 + 25 n4 + 5 n6 + n8 (the 35 mixes of
// four blocks).
template <int C>
bool dispatch_few(int code, const AttnPagedArgs &a, int splits, unsigned wgs, hipStream_t s) {
  constexpr int n3 = C / 125, n4 = C / 25 % 5, n6 = C / 5 % 5, n8 = C % 5;
  if constexpr (n3 + n4 + n6 + n8 == 4) {
    if (code == C) {
      using Mx = Mix<n3, n4, n6, n8>;
      const auto fn = a.o_f32 ? attn_few_kernel<true, Mx> : attn_few_kernel<false, Mx>;
      hipLaunchKernelGGL(fn, dim3(wgs), dim3(64 * kFewWaves), 0, s, a, splits);
      return true;
    }
  }
  if constexpr (C > 0) {
    return dispatch_few<C - 1>(code, a, splits, wgs, s);
  } else {
    return false;
  }
}

int64_t tile_numbers(const AttnPagedArgs &a) { return a.T * a.G / kRows + a.S; }

// Splits of each kernel, 0 where it is not launched.
struct Plan {
  int tile, few;
};
Plan plan_of(const AttnPagedArgs &a) {
  Plan p = {0, 0};
  const int64_t Hkv = a.geo.Hkv;
  auto split = [](int64_t wgs, int64_t want, int64_t steps, int64_t least) {
    const int64_t n = std::min(want / std::max<int64_t>(wgs, 1), steps / least);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, kMaxSplits));
  };
  // every sequence has max_q rows where their sum says so
  if (a.max_q * a.G > kFewRows)
    p.tile = split(tile_numbers(a) * Hkv, 1024, (a.max_kv + kTok - 1) / kTok, 4);
  if (a.max_q * a.G <= kFewRows || (a.G <= kFewRows && a.T < a.S * a.max_q))
    p.few = split(a.S * Hkv, 1024, (a.max_kv + kChunk - 1) / kChunk, kFewWaves);
  return p;
}

}  // namespace

int64_t attn_paged_work(const AttnPagedArgs &a) {
  const Plan p = plan_of(a);
  const int n = std::max(p.tile, p.few);
  return n <= 1 ? 0 : n * a.T * a.Hq * (kD + 2) * (int64_t)sizeof(float);
}

hipError_t launch_attn_paged(const AttnPagedArgs &args, hipStream_t s) {
  AttnPagedArgs a = args;
  const Plan p = plan_of(a);
  a.parts = std::max(p.tile, p.few);
  const int64_t numbers = tile_numbers(a);
  const int64_t wgs = numbers * a.geo.Hkv * p.tile, few_wgs = a.S * a.geo.Hkv * p.few;
  // (a dispatch holds fewer than 2^32 threads)
  if (std::max(wgs, few_wgs) >= ((int64_t)1 << 32) / 256) return hipErrorInvalidValue;
  if (p.few) {
    int n[9] = {};
    for (int b = 0; b < 4; ++b) ++n[a.geo.m[b]];
    if (!dispatch_few<500>(125 * n[3] + 25 * n[4] + 5 * n[6] + n[8], a, p.few, (unsigned)few_wgs, s))
      return hipErrorInvalidValue;
  }
  if (p.tile) {
    const auto fn = a.o_f32 ? attn_tile_kernel<true> : attn_tile_kernel<false>;
    hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(64 * kWaves), 0, s, a, p.tile, numbers,
                       p.few ? 1 : 0);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts <= 1) return e;
  const auto merge = a.o_f32 ? attn_merge_kernel<true> : attn_merge_kernel<false>;
  hipLaunchKernelGGL(merge, dim3((unsigned)((a.T * a.Hq + 7) / 8)), dim3(256), 0, s, a,
                     p.tile ? p.tile : p.few, p.few ? p.few : p.tile);
  return hipGetLastError();
}

}  // namespace mxq
