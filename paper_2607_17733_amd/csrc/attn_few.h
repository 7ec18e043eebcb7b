// attn_few.h -- attention over the paged cache for sequences with few query rows
// (decoding, drafted tokens): the kernel, instantiated for float32 and for bf16
// results by one source each.
//
// Bytes and their dequantization bound it, not products.  Each wave takes chunks of
// 32 tokens by itself, without a barrier: K is dequantized straight into the operand
// of 16x16x32 products, S^T = K Q^T with a lane per query row, V into the wave's own
// LDS rows, from where the transposing read brings it to O^T += V^T P^T.  The next
// chunk's packed rows are on their way while one is computed, in a second set of
// registers, and its pages' numbers another chunk ahead.  The waves, then the
// splits, are merged in a fixed order.  Each width mix is its own instance, so block
// offsets and widths are compile-time constants: with widths looked up the loop had
// 147 waits for loads, and 32 sequences of 2048 to 8192 tokens of 4/4/6/8 bits went from
// 193 to 88 us (80 now).
#pragma once

#include "attn_paged_device.h"

namespace mxq {

namespace {

constexpr int kFewWaves = 4;
// LDS rows of a wave's 32 dequantized V tokens: the stride puts the rows of eight lanes'
// 16-byte writes, and of a transposing read, into distinct banks, and every access is
// a base plus a constant.
constexpr int kFewRow = kRowBytes + 32;
constexpr int kFewBytes = kFewChunk * kFewRow;

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

// A lane's place in the planes of a page, for the page's token i + n: at[j] + 4 m_j i
// (rows of one width: at[0]).
template <class Mx>
struct Place {
  uint32_t at[4];
};
template <class Mx>
__device__ __forceinline__ Place<Mx> place_of(int lg_page, int g, int n) {
  Place<Mx> p;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    constexpr int kM0 = Mx::width(0);
    const int m = Mx::width(j);
    p.at[j] = Mx::kUniform ? ((uint32_t)(4 * kM0 * g) << lg_page) + n * 4 * kM0
                           : ((uint32_t)Mx::off(j) << lg_page) + n * 4 * m +
                                 (m == 8 ? 8 * g : m == 3 ? ((3 * g) & ~3) : 4 * g);
  }
  return p;
}
// `page`: the page's first token of the head, with 16 tokens from token i on.
template <class Mx, int J>
__device__ __forceinline__ void load_group(const uint8_t *page, uint32_t i, const Place<Mx> &pl, int g,
                                           RawRow<Mx> &r) {
  constexpr int M = Mx::width(J), S = Mx::start(J);
  const uint8_t *p = page + i * (4 * M) + pl.at[J];
  r.w[S] = *(const uint32_t *)p;
  if constexpr (M == 6) {                // low nibbles, and the half block's top bits
    r.w[S + 1] = *(const uint32_t *)(page + i * (4 * M) + pl.at[J] + 16 - 4 * g + 4 * (g >> 1));
  } else if constexpr (M == 8) {
    r.w[S + 1] = *(const uint32_t *)(p + 4);
  } else if constexpr (M == 3) {         // bytes 3 g .. 3 g + 2 of twelve
    r.w[S + 1] = *(const uint32_t *)(p + (g < 3 ? 4 : 0));
  }
}
template <class Mx>
__device__ __forceinline__ void load_row(const uint8_t *page, uint32_t i, const Place<Mx> &pl, int g,
                                         RawRow<Mx> &r) {
  if constexpr (Mx::kUniform) {
    constexpr int M = Mx::width(0);
    RawBlock b;
    load_block<M>(page + i * (4 * M) + pl.at[0], b);
#pragma unroll
    for (int k = 0; k < M; ++k) r.w[k] = b.w[k];
  } else {
    load_group<Mx, 0>(page, i, pl, g, r);
    load_group<Mx, 1>(page, i, pl, g, r);
    load_group<Mx, 2>(page, i, pl, g, r);
    load_group<Mx, 3>(page, i, pl, g, r);
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

// Nonzero if one of four exponents may pass max_exp (E >= 224).
__device__ inline uint32_t big_bits(uint32_t ex) { return ex & (ex << 1) & (ex << 2) & 0x80808080u; }

__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A lane's packed rows of a chunk: tokens 16 mt + n.  hole: a half whose page is none.
template <class Mx>
struct Chunk {
  RawRow<Mx> k[2], v[2];
  bool hole[2];
};

// Waves per SIMD that two sets of a chunk's registers leave room for, by the groups of
// 16 query rows and a lane's words of a row.
constexpr int few_waves(int groups, int words) {
  return groups > 1 || words > 6 ? 2 : words > 4 ? 3 : 4;
}

// NC: groups of 16 query rows.
template <bool F32, class Mx, int NC>
__global__ __launch_bounds__(64 * kFewWaves, few_waves(NC, Mx::kWords))
void attn_few_kernel(AttnPagedArgs a, int splits) {
  __shared__ __attribute__((aligned(16))) uint8_t pool[kFewWaves][kFewBytes];
  __shared__ float mm[kFewWaves][16 * NC], ml[kFewWaves][16 * NC];
  const PageGeo &g = a.geo;
  const int t = threadIdx.x, lane = t & 63, gr = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint32_t Hkv = (uint32_t)g.Hkv;
  const int G = a.G;
  // KV heads run fastest, then a sequence's splits (32 sequences of 2048 to 8192 tokens of
  // 4/4/6/8 bits: 80 us; sequences before splits 89, heads last 91)
  const uint32_t rest = blockIdx.x / Hkv;
  const int kvh = (int)(blockIdx.x - rest * Hkv);
  const int s = (int)(rest / (uint32_t)splits), split = (int)(rest - (uint32_t)s * (uint32_t)splits);
  const Seq q = seq_at(a, s);
  if (q.n == 0 || (int64_t)q.n * G > 16 * NC) return;
  const int rows = q.n * G;
  const int p0 = q.p0;
  const Steps st = steps_of<kFewChunk>(a, q, p0, (int64_t)p0 + q.n - 1);
  const int v0 = (int)((int64_t)st.count * split / splits);
  const int v1 = (int)((int64_t)st.count * (split + 1) / splits);

  // A chunk's halves of 16 tokens lie in one page each (a half past the last token is
  // the chunk's first).  Places past the last token are read too, they are the page's
  // own, and are cleared where they are used.
  const int32_t *pages = a.table + (int64_t)s * a.ld_table;
  const int page_mask = (1 << g.lg_page) - 1, last = q.len - 1;
  // (past the last chunk: the last one)
  auto first_of = [&](int v) {
    const int u = min(v, v1 - 1);
    return (u < st.pre ? u : u + st.shift) * kFewChunk;
  };
  auto half_of = [&](int t0, int mt) { return t0 + 16 * mt <= last ? t0 + 16 * mt : t0; };
  int pg[2];
  auto number = [&](int v) __attribute__((always_inline)) {
    const int t0 = first_of(v);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) pg[mt] = pages[half_of(t0, mt) >> g.lg_page];
  };
  const uint32_t page_rows = Hkv << g.lg_page;             // rows of a page, below 2^26
  const Place<Mx> place = place_of<Mx>(g.lg_page, gr, n);
  auto fetch = [&](int v, Chunk<Mx> &c) __attribute__((always_inline)) {
    const int t0 = first_of(v);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      c.hole[mt] = (uint32_t)pg[mt] >= (uint32_t)g.pages;
      const uint32_t page = c.hole[mt] ? 0u : (uint32_t)pg[mt];
      const int64_t run = (int64_t)((uint64_t)page * page_rows + ((uint32_t)kvh << g.lg_page));
      const uint32_t i = (uint32_t)(half_of(t0, mt) & page_mask);
      const int64_t at = run * g.row;
      load_row<Mx>(a.k_mant + at, i, place, gr, c.k[mt]);
      load_row<Mx>(a.v_mant + at, i, place, gr, c.v[mt]);
      c.k[mt].ex = *(const uint32_t *)(a.k_exp + (run + i) * 4 + 4 * n);
      c.v[mt].ex = *(const uint32_t *)(a.v_exp + (run + i) * 4 + 4 * n);
    }
  };
  Chunk<Mx> c0, c1;
  int v = v0 + wave;
  if (v < v1) {
    number(v);
    fetch(v, c0);
    number(v + kFewWaves);
  }

  // this lane's query rows (columns past the last repeat it); product j of a score
  // takes the values of lane group gr, in slot order
  const int window = (int)(a.window && a.window < INT32_MAX ? a.window : INT32_MAX);
  const float sc = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * (a.softcap.cap > 0.f ? 1.f : kUnit<F32>);
  const float ninf = -__builtin_inff();
  bf8 qop[NC][4];
  float slope[NC], m[NC], ref[NC], l[NC];
  int p[NC];
  f4 o[NC][8];                                             // row n, slots 16 dt + 4 gr ..
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int r = min(16 * c + n, rows - 1), tok = r / G, hd = kvh * G + r - tok * G;
    const uint16_t *src = a.q + (int64_t)(q.row0 + tok) * a.q_ts + hd * a.q_hs;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u4 w = *(const u4 *)(src + Mx::value(gr, j));
      w = a.scale == 0.f ? u4{0u, 0u, 0u, 0u} : w ^ u4{sign, sign, sign, sign};
      if (split_slots(Mx::width(j)))
        w = u4{__builtin_amdgcn_perm(w[1], w[0], 0x05040100), __builtin_amdgcn_perm(w[3], w[2], 0x05040100),
               __builtin_amdgcn_perm(w[1], w[0], 0x07060302), __builtin_amdgcn_perm(w[3], w[2], 0x07060302)};
      qop[c][j] = __builtin_bit_cast(bf8, w);
    }
    slope[c] = a.slopes ? a.slopes[hd] * kUnit<F32> : 0.f;
    p[c] = p0 + tok;
    m[c] = ninf;
    ref[c] = l[c] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[c][dt] = f4{0.f, 0.f, 0.f, 0.f};
  }
  uint8_t *vs = pool[wave];
  uint8_t *const vw = vs + n * kFewRow + 2 * Mx::value(gr, 0);
  const uint8_t *const vr = vs + (4 * gr + (n >> 2)) * kFewRow + 8 * (n & 3);

  auto compute = [&](int v, Chunk<Mx> &c) __attribute__((always_inline)) {
    const int t0 = first_of(v);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
      if (c.hole[mt]) {                                    // zero rows
#pragma unroll
        for (int k = 0; k < Mx::kWords; ++k) c.k[mt].w[k] = c.v[mt].w[k] = 0u;
        c.k[mt].ex = c.v[mt].ex = 0u;
      }
    if (t0 > q.len - kFewChunk) {                          // places past the last token: tiny values
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
        if (t0 + 16 * mt + n > last) c.k[mt].ex = c.v[mt].ex = 0u;
    }
    const bool big = __any((big_bits(c.k[0].ex) | big_bits(c.k[1].ex) | big_bits(c.v[0].ex) |
                            big_bits(c.v[1].ex)) != 0);
    // scores: tokens 16 mt + 4 gr + i of row n
    f4 sa[NC][2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      bf8 k[4];
      dequant_row(c.k[mt], gr, big, k);
#pragma unroll
      for (int e = 0; e < NC; ++e) {
        sa[e][mt] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          sa[e][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], qop[e][j], sa[e][mt], 0, 0, 0);
      }
    }
    wave_sync();                                           // the last chunk's V rows are consumed
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      bf8 w[4];
      dequant_row(c.v[mt], gr, big, w);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(bf8 *)(vw + 16 * mt * kFewRow + 2 * (Mx::value(0, j) - Mx::value(0, 0))) = w[j];
    }
    wave_sync();
    constexpr int kTerms = F32 ? 3 : 1;
    bf8 pt[NC][kTerms];
    // (positions end before the sequence does, and so does the prefix)
    const bool edge = t0 + kFewChunk - 1 > p0 || last - t0 >= window;
#pragma unroll
    for (int e = 0; e < NC; ++e) {
      float x[8];                                          // the product's slots: tokens 4 gr + i, 16 + 4 gr + i
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = sa[e][i >> 2][i & 3];
      float scale = sc;
      if (a.softcap.cap > 0.f) {
        cap_scores<F32, 8>(x, sc, a.softcap.cap, a.softcap.k, a.softcap.two);
        scale = 1.f;
      }
      if (a.slopes) {
        const float rel = (float)(p[e] - t0 - 4 * gr);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = fmaf(-slope[e], fabsf(rel - (float)(16 * (i >> 2) + (i & 3))), x[i] * scale);
        scale = 1.f;
      }
      if (edge) {
        const int rel = p[e] - t0 - 4 * gr, pre = q.pre - t0 - 4 * gr;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = 16 * (i >> 2) + (i & 3);
          const bool see = ((uint32_t)(rel - k) < (uint32_t)window) | (k < pre);
          x[i] = see ? x[i] : ninf;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                        fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      top = top == ninf ? ninf : top * scale;
      if (__any(top > m[e] + kSlack<F32> || (m[e] == ninf && top != ninf))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float nm = fmaxf(m[e], top);
        const float alpha = m[e] == ninf ? 0.f : weight<F32>(m[e] - nm);
        m[e] = nm;
        ref[e] = nm == ninf ? 0.f : nm;                    // scores of -inf weigh 0
        l[e] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[e][dt] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = weight<F32>(fmaf(x[i], scale, -ref[e]));
        if constexpr (F32) l[e] += x[i];
      }
#pragma unroll
      for (int k = 0; k < kTerms; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          pt[e][k][i] = (__bf16)x[i];
          if constexpr (F32) x[i] -= (float)pt[e][k][i];
        }
      if constexpr (!F32) {                                // the sum of what the values are weighted with
#pragma unroll
        for (int i = 0; i < 8; i += 2)
          l[e] = __builtin_amdgcn_fdot2_f32_bf16(bf2{pt[e][0][i], pt[e][0][i + 1]},
                                                 bf2{(__bf16)1.f, (__bf16)1.f}, l[e], false);
      }
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(vr + 32 * dt));
      const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(vr + 32 * dt + 16 * kFewRow));
      const bf8 vv = __builtin_bit_cast(bf8, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int e = 0; e < NC; ++e)
#pragma unroll
        for (int k = 0; k < kTerms; ++k)
          o[e][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pt[e][k], o[e][dt], 0, 0, 0);
    }
  };
  // The next chunk's rows are asked for before one is computed, then the page numbers
  // of the one after it.  (Also behind the last chunk: a load under a condition would
  // make the compiler wait for all of them where one set's rows are used.)
  auto step = [&](Chunk<Mx> &cur, Chunk<Mx> &next) __attribute__((always_inline)) {
    fetch(v + kFewWaves, next);
    number(v + 2 * kFewWaves);
    compute(v, cur);
    v += kFewWaves;
  };
  while (v < v1) {
    step(c0, c1);
    if (v >= v1) break;
    step(c1, c0);
  }
  // Merge the waves in order: each writes its outputs, weighted against the row's
  // largest reference, over its V rows (four values at a time xor the row: sixteen
  // rows' writes lie in distinct banks).
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
    if (gr == 0) {
      mm[wave][16 * c + n] = m[c];
      ml[wave][16 * c + n] = l[c];
    }
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float M = ninf;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) M = fmaxf(M, mm[w][16 * c + n]);
    const float f = m[c] == ninf ? 0.f : weight<F32>(m[c] - M);
    float *mo = (float *)vs;                               // [row][d]
    if (c > 0) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const int d8 = 16 * dt + 8 * (gr >> 1);
      const bool sp = split_slots(Mx::width(dt >> 1));
#pragma unroll
      for (int i = 0; i < 4; ++i)                          // (0 without a finite score; a NaN stays)
        mo[n * kD + ((d8 + (sp ? 2 * i + (gr & 1) : 4 * (gr & 1) + i)) ^ 4 * n)] = o[c][dt][i] * f;
    }
    __syncthreads();
    const int here = min(rows - 16 * c, 16);
    for (int i = t; i < here * (kD / 4); i += 64 * kFewWaves) {
      const int row = i / (kD / 4), d = 4 * (i % (kD / 4)), r = 16 * c + row;
      float M2 = ninf, L = 0.f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) M2 = fmaxf(M2, mm[w][r]);
      f4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        L += mm[w][r] == ninf ? ml[w][r] : ml[w][r] * weight<F32>(mm[w][r] - M2);
        O += *(const f4 *)((float *)pool[w] + row * kD + (d ^ 4 * row));
      }
      const int tk = r / G;
      const int64_t at = (int64_t)(q.row0 + tk) * a.Hq + kvh * G + r - tk * G;
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
}

// The kernel for a row's widths, code = 125 n3 + 25 n4 + 5 n6 + n8 (the 35 mixes of
// four blocks).
template <bool F32, int C>
bool dispatch_few(int code, const AttnPagedArgs &a, int splits, int groups, hipStream_t s) {
  constexpr int n3 = C / 125, n4 = C / 25 % 5, n6 = C / 5 % 5, n8 = C % 5;
  if constexpr (n3 + n4 + n6 + n8 == 4) {
    if (code == C) {
      using Mx = Mix<n3, n4, n6, n8>;
      const auto fn = groups == 1 ? attn_few_kernel<F32, Mx, 1> : attn_few_kernel<F32, Mx, 2>;
      hipLaunchKernelGGL(fn, dim3((unsigned)(a.S * a.geo.Hkv * splits)), dim3(64 * kFewWaves), 0, s,
                         a, splits);
      return true;
    }
  }
  if constexpr (C > 0) {
    return dispatch_few<F32, C - 1>(code, a, splits, groups, s);
  } else {
    return false;
  }
}

template <bool F32>
hipError_t launch_few(const AttnPagedArgs &a, int splits, int groups, hipStream_t s) {
  int n[9] = {};
  for (int b = 0; b < 4; ++b) ++n[a.geo.m[b]];
  if (!dispatch_few<F32, 500>(125 * n[3] + 25 * n[4] + 5 * n[6] + n[8], a, splits, groups, s))
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace
}  // namespace mxq
