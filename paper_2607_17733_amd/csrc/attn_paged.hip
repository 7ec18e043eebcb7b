// attn_paged.hip -- attention of new tokens over the paged MXINT KV cache
// (include/mxq.h states the operation).
//
// A sequence's n new tokens and the G query heads of a KV head make n G query
// rows that share K and V (row r: token r / G, head r % G).  A workgroup takes a
// tile of them, 32 a wave, and walks the cached tokens, 64 at a time, with a
// running maximum and sum of the softmax (one pass over K and V):
//   S^T = K Q^T     32x32x16 bf16 products, a lane holding one query row's scores
//                   of 16 of the 32 tokens (its partner, lane ^ 32, the others);
//   O^T += V^T P^T  takes the same lane's probabilities as they come out of the
//                   softmax: the order of the tokens over the reduction is free,
//                   and V follows it.
// So the statistics and the rescaling of O are a lane's own, and P never leaves
// the registers.  K and V are dequantized once per workgroup into LDS as bf16,
// which is exact (at most 8 significant bits): a wave per 32-value block of the
// row, a lane per token, so that widths are uniform over a wave.  What arrives in
// LDS by one barrier is V's step and K's half a step further, so that each half
// step has the next one's score products to put its exponentials behind.
//
// A step's 32 products of a wave hold its matrix core for 1024 cycles; behind them
// go the exponentials, the sums and the dequantization, about as many issue cycles.
// 2048 tokens over 16384, 64 query and 8 KV heads, 4-bit: 1040 us, 0.99 PFLOP/s
// (1.24 to 1.37 by a large library product), the matrix cores 41 % and the vector
// units 55 % busy by the counters: softmax and dequantization bound it.
// For a bf16 result the probabilities enter the second product rounded to bf16 (the
// result is then 0.0018 to 0.0022 off the exact one, 0.0017 of it its own rounding), for
// a float32 one as three bf16 terms, which are they exactly: 1945 us.
//
// Sequences with few query rows per KV head (decoding, drafted tokens) have a kernel of
// their own (attn_few.h): up to 32 where no sequence of the batch has more, beside tiles
// up to 16 (32 with 17 to 32 query heads per KV head).  The tokens of a sequence are split over
// workgroups where there are few rows; the splits' results are merged in order.
#include <algorithm>

#include "attn_paged_device.h"

namespace mxq {

namespace {

constexpr int kTok = 64;                 // tokens per step
constexpr int kFewMost = 32;             // query rows of the kernel for few
constexpr int kMaxSplits = 256;

// LDS rows of a token's 128 bf16 values.  The strides put sixteen tokens' operand
// reads of K, and a transposing read of V (four tokens, 64 bytes), into distinct banks;
// every access is a base plus a constant (an exclusive-or swizzle costs twenty
// address registers, which the loop does not have).
constexpr int kKRow = kRowBytes + 16, kVRow = kRowBytes + 64;
constexpr int kKBytes = kTok * kKRow, kVBytes = kTok * kVRow, kStage = kKBytes + kVBytes;

// Keeps the packed words packed until here: the conversions that the ways to dequantize
// a block have in common would else be done when it is loaded, and held in 32 registers.
template <int M>
__device__ __forceinline__ RawBlock packed(const RawBlock &r) {
  RawBlock b;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    b.w[i] = r.w[i];
    asm volatile("" : "+v"(b.w[i]));
  }
  return b;
}

// A token's block to its place in LDS, without the rest of the scale that blocks beyond
// max_exp have ...
template <int M>
__device__ __forceinline__ void store_block(const RawBlock &r, int E, uint8_t *to) {
  const RawBlock b = packed<M>(r);
#pragma unroll
  for (int j = 0; j < 4; ++j) *(bf8 *)(to + 16 * j) = dequant8<M>(b, j, E);
}
// ... and again with it.
template <int M>
__device__ __forceinline__ void store_big(const RawBlock &r, int E, uint8_t *to) {
  const RawBlock b = packed<M>(r);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bf8 v = dequant8<M>(b, j, E);
    big_scale<M>(v, E);
    *(bf8 *)(to + 16 * j) = v;
  }
}

// The sum of the lanes up to this one.
__device__ inline int wave_scan(int x, int lane) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // shifts within 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  const int r0 = __builtin_amdgcn_readlane(x, 15), r1 = __builtin_amdgcn_readlane(x, 31),
            r2 = __builtin_amdgcn_readlane(x, 47);
  return x + (lane >= 16 ? r0 : 0) + (lane >= 32 ? r1 : 0) + (lane >= 48 ? r2 : 0);
}

// Tile `index` of the sequences with more than few_rows query rows, ROWS rows each, a
// sequence's last first.  The launch has floor(T G / ROWS) + S tiles, which are enough
// without a look at the device's lengths (n rows have at most floor(end / ROWS) -
// floor(begin / ROWS) + 1).  Up to 64 sequences are counted, in one load latency, and the
// tiles too many come last (among the others, say every second one, they leave half of
// the GPU idle: workgroups are dealt to its parts in turn; 16 sequences of 256 rows over
// 2000 tokens, 102 us).  More have their numbers with gaps, those of sequence s from
// floor(cu_q[s] G / ROWS) + s on, found by 64-way search.  False: none.
template <int ROWS>
__device__ inline bool find_tile(const AttnPagedArgs &a, int64_t index, int64_t tiles, int few_rows, Seq &q,
                                 int &tile) {
  const int lane = threadIdx.x & 63, S = (int)a.S;
  auto start = [&](int s, int cu) { return (int64_t)max(cu, 0) * a.G / ROWS + s; };
  int64_t number = tiles - 1 - index;
  int lo = 0, cnt = S;
  while (cnt > 64) {
    const int step = (cnt + 63) / 64, s = lo + lane * step;
    const bool le = s < lo + cnt && start(s, a.cu_q[min(s, S)]) <= number;
    const int k = __popcll(__ballot(le));
    if (k == 0) return false;
    lo += (k - 1) * step;
    cnt = min(step, S - lo);
  }
  const int s = min(lo + lane, S - 1);
  const Seq x = seq_at(a, s);
  const int64_t r = (int64_t)x.n * a.G;
  int k, first;
  if (S <= 64) {
    const int n = lane < S && r > few_rows ? (int)((r + ROWS - 1) / ROWS) : 0, end = wave_scan(n, lane);
    number = __builtin_amdgcn_readlane(end, 63) - 1 - index;
    if (number < 0) return false;
    k = __popcll(__ballot(end <= number));
    first = __builtin_amdgcn_readlane(end - n, k);
  } else {
    const int at = (int)start(s, a.cu_q[s]);
    k = __popcll(__ballot(lane < cnt && at <= number)) - 1;
    if (k < 0) return false;
    first = __builtin_amdgcn_readlane(at, k);
  }
  q.s = lo + k;
  q.row0 = __builtin_amdgcn_readlane(x.row0, k);
  q.n = __builtin_amdgcn_readlane(x.n, k);
  q.p0 = __builtin_amdgcn_readlane(x.p0, k);
  q.len = __builtin_amdgcn_readlane(x.len, k);
  q.pre = __builtin_amdgcn_readlane(x.pre, k);
  tile = (int)(number - first);
  return true;
}

// A wave's share of a tile: 32 query rows, a row per lane and its partner.
struct TileRow {
  int p;                                 // the row's position
  int pw0, pw1;                          // the wave's first and last
  int last;                              // the last token that one of the wave's rows may see
  int window, pre;
  float sc, slope, cap, cap_k;
  bool biased;
};

// S^T of half a step: 32 tokens (`rows`: row x, 16 h bytes on), this lane's query row;
// value i is token 4 h + 8 (i / 4) + i % 4.
__device__ __forceinline__ bf8 k_operand(const uint8_t *rows, int ks) {
  return *(const bf8 *)(rows + 32 * ks);
}
__device__ __forceinline__ void scores(const uint8_t *rows, const bf8 (&qop)[8], f16v &s) {
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int ks = 0; ks < 8; ++ks)
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(rows, ks), qop[ks], s, 0, 0, 0);
}
// V^T operand of product i of half a step: tokens 16 (i / 4) .., values 32 (i % 4) ..;
// lane half h holds its tokens 4 h .. 4 h + 3 and 8 + 4 h ..
__device__ __forceinline__ bf8 v_operand(const uint8_t *vt, int i) {
  const uint8_t *at = vt + 16 * (i >> 2) * kVRow + 64 * (i & 3);
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)at);
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(at + 8 * kVRow));
  return __builtin_bit_cast(bf8, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Caps, biases and masks of half a step from token t0 on; returns the factor that is
// left to apply.
template <bool F32>
__device__ __forceinline__ float adjust(const TileRow &w, int t0, int h, f16v &s) {
  auto c = [](int i) { return 8 * (i >> 2) + (i & 3); };
  float scale = w.sc;
  if (w.cap > 0.f) {
    cap_scores<F32, 16>(s, scale, w.cap, w.cap_k, -2.f * w.cap);
    scale = 1.f;
  }
  if (w.biased) {
    const float rel = (float)(w.p - t0 - 4 * h);
    if (t0 + 31 > w.pw0 && w.pre > 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = fmaf(-w.slope, fabsf(rel - (float)c(i)), s[i] * scale);
    } else {                                               // (no token behind its row is visible)
      const float near = -w.slope * rel;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale, fmaf(w.slope, (float)c(i), near));
    }
    scale = 1.f;
  }
  // Masks, where not every row of the wave sees all.  (Positions end before the
  // sequence does, and so does the prefix: its length needs no test.)
  if (t0 + 31 > w.pw0 || w.pw1 - t0 >= w.window) {
    const int rel = w.p - t0 - 4 * h, pre = w.pre - t0 - 4 * h;
    if (w.pre > t0) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[i] = (uint32_t)(rel - c(i)) < (uint32_t)w.window || c(i) < pre ? s[i] : -__builtin_inff();
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[i] = (uint32_t)(rel - c(i)) < (uint32_t)w.window ? s[i] : -__builtin_inff();
    }
  }
  return scale;
}

// Dequantization: a wave's block of a step's K or V rows, a lane per token.  V's
// unit v are the tokens of step v; K's are the second half of step v and the first
// half of step v + 1.
struct Loader {
  const int32_t *pages;                  // of the sequence
  int64_t plane;                         // of the block, in a page of one head
  uint32_t page_rows, head_rows;         // rows of a page; those of the heads before
  int blk, lane, last, lg_page, row, n_pages;
  Steps st;
  int v1;
  // (past the last step: the last step's)
  __device__ __forceinline__ int token(int v, bool k) const {
    const int at = lane + (k ? kTok / 2 : 0);
    const int u = min(max(v + (at >> 6), 0), v1 - 1);
    return min((u < st.pre ? u : u + st.shift) * kTok + (at & (kTok - 1)), last);
  }
  __device__ __forceinline__ int page(int v, bool k) const { return pages[token(v, k) >> lg_page]; }
  // The packed block and its exponent; false for a page outside the pool.
  template <int M>
  __device__ __forceinline__ bool load(const uint8_t *mant, const uint8_t *exp, int v, bool k, int page,
                                       RawBlock &r, uint32_t &E) const {
    const bool hole = (uint32_t)page >= (uint32_t)n_pages;
    const uint32_t i = (uint32_t)token(v, k) & ((1u << lg_page) - 1);
    const int64_t run = (int64_t)((uint64_t)(hole ? 0u : (uint32_t)page) * page_rows + head_rows);
    load_block<M>(mant + run * row + plane + i * (4 * M), r);
    E = exp[(run + i) * 4 + blk];
    return !hole;
  }
};

// A unit's block to LDS, where it needs more than store_block: pages outside the pool
// (zero rows), exponents beyond max_exp.
template <int M>
__device__ __forceinline__ void store_rest(RawBlock &r, uint32_t E, bool good, uint8_t *to) {
  if (__any(!good || (int)E > max_exp(M))) {
#pragma unroll
    for (int k = 0; k < 8; ++k) r.w[k] = good ? r.w[k] : 0u;
    store_big<M>(r, (int)E, to);
  }
}

// Half a step: the probabilities of its 32 tokens while the next half's scores are
// computed, then its share of the values while GROUPS groups of a packed block, from G0
// on, are dequantized.
// A product holds the matrix core for 32 cycles, in which the wave issues eight vector
// instructions: the work is cut into eight pieces each and one put behind each product,
// in this order (left to itself the compiler puts the products in a row: every
// sched_barrier keeps it from that), operands read two products ahead.
template <bool F32, int M, int G0, int GROUPS>
__device__ __forceinline__ void half_step(const TileRow &w, int t0, int h, const bf8 (&qop)[8],
                                          const uint8_t *next_rows, const uint8_t *vt, f16v &s, f16v &nx,
                                          f16v (&o)[4], float &m, float &ref, float &l, RawBlock &r,
                                          uint32_t E, uint8_t *to) {
  const float ninf = -__builtin_inff();
  bf8 kop[2] = {k_operand(next_rows, 0), k_operand(next_rows, 1)}, vop[2];
  const float scale = adjust<F32>(w, t0, h, s);
  float top = s[0];
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
  top = fmaxf(top, other_half(top));
  top = top == ninf ? ninf : top * scale;
  if (__any(top > m + kSlack<F32> || (m == ninf && top != ninf))) {
    const float nm = fmaxf(m, top);
    const float alpha = m == ninf ? 0.f : weight<F32>(m - nm);
    m = nm;
    ref = nm == ninf ? 0.f : nm;                           // scores of -inf weigh 0
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) nx[i] = 0.f;
  constexpr int kTerms = F32 ? 3 : 1;
  bf8 pt[2][kTerms];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    nx = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[i & 1], qop[i], nx, 0, 0, 0);
    if (i < 6) kop[i & 1] = k_operand(next_rows, i + 2);
    else vop[i & 1] = v_operand(vt, i - 6);
    float e0 = weight<F32>(fmaf(s[2 * i], scale, -ref)), e1 = weight<F32>(fmaf(s[2 * i + 1], scale, -ref));
    if constexpr (F32) l += e0 + e1;
#pragma unroll
    for (int k = 0; k < kTerms; ++k) {
      const bf2 y = {(__bf16)e0, (__bf16)e1};
      if constexpr (!F32) l = __builtin_amdgcn_fdot2_f32_bf16(y, bf2{(__bf16)1.f, (__bf16)1.f}, l, false);
      pt[i >> 2][k][2 * (i & 3)] = y[0];
      pt[i >> 2][k][2 * (i & 3) + 1] = y[1];
      if constexpr (F32) {
        e0 -= (float)y[0];
        e1 -= (float)y[1];
      }
    }
  }
  const RawBlock b = packed<M>(r);
  const float sc = factor<M>((int)E);
  Ints u = {0, 0};
  bf4 first = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kTerms; ++k)
      o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop[i & 1], pt[i >> 2][k], o[i & 3], 0, 0, 0);
    if (i < 6) vop[i & 1] = v_operand(vt, i + 2);
    // (4-bit integers take twice as long as their conversion)
    constexpr int kPer = 8 / GROUPS;                       // products per group
    const int j = G0 + i / kPer;
    if (i % kPer == 0) {
      u = ints8<M>(b, j);
      if constexpr (M != 4) first = four<M>(u.b0, sc);
    } else if (i % kPer == kPer / 2) {
      if constexpr (M == 4) first = four<M>(u.b0, sc);
      *(bf8 *)(to + 16 * j) = both(first, four<M>(u.b1, sc));
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}

// The steps v0 .. v1 - 1 of a tile, for a wave whose block has M bits.  One barrier
// per step: behind it K's unit v and V's unit v are in LDS, and nobody reads the
// other buffers any more, which take the units v + 1 meanwhile.  Four waves dequantize
// a block of K and one of V each, of eight the first four one of K, the others one of V
// (job_k: which).  `live`: the wave has query rows; where it has none, or none that see
// the step, it only dequantizes.
template <bool F32, int NW, int M>
__device__ __forceinline__ void tile_steps(const AttnPagedArgs &a, const Loader &ld, int v0, int v1,
                                           bool job_k, bool live, const TileRow &w, const bf8 (&qop)[8],
                                           uint8_t *lds, f16v (&o)[4], float &m, float &l) {
  const int lane = ld.lane, h = lane >> 5, n = lane & 15;
  // where this lane reads K's and V's operands and writes its blocks
  const int kr = (lane & 31) * kKRow + 16 * h;
  const int vr = kKBytes + (4 * h + (n >> 2)) * kVRow + 32 * (lane >> 4 & 1) + 8 * (n & 3);
  const int kw = lane * kKRow + 64 * ld.blk, vw = kKBytes + lane * kVRow + 64 * ld.blk;
  const bool k1 = NW == 4 || job_k;                        // the first block's job
  const int w1 = k1 ? kw : vw;
  RawBlock r1, r2;
  uint32_t e1, e2;
  bool g1, g2;                                             // (false: the page is outside the pool)
  const uint8_t *const m1 = k1 ? a.k_mant : a.v_mant, *const x1 = k1 ? a.k_exp : a.v_exp;
  auto load_1 = [&](int v, int page) { g1 = ld.template load<M>(m1, x1, v, k1, page, r1, e1); };
  auto load_2 = [&](int v, int page) { g2 = ld.template load<M>(a.v_mant, a.v_exp, v, false, page, r2, e2); };
  auto put = [&](RawBlock &r, uint32_t E, bool good, uint8_t *to) {
    store_block<M>(r, (int)E, to);
    store_rest<M>(r, E, good, to);
  };
  // K's units v0 - 1 (its second half is the first step's first) and v0, V's unit v0,
  // all their loads in flight together, then those of the units v0 + 1
  uint8_t *cur = lds, *nxt = lds + kStage;
  int n1 = ld.page(v0, k1), n2 = NW == 4 ? ld.page(v0, false) : 0;
  const int p0 = ld.page(v0 - 1, true), p1 = ld.page(v0 + 1, k1), p2 = NW == 4 ? ld.page(v0 + 1, false) : 0;
  RawBlock r0;
  uint32_t e0 = 0;
  bool g0 = true;
  if (k1) g0 = ld.template load<M>(a.k_mant, a.k_exp, v0 - 1, true, p0, r0, e0);
  load_1(v0, n1);
  if constexpr (NW == 4) load_2(v0, n2);
  n1 = ld.page(v0 + 2, k1);
  if constexpr (NW == 4) n2 = ld.page(v0 + 2, false);
  if (k1) put(r0, e0, g0, nxt + kw);
  put(r1, e1, g1, cur + w1);
  load_1(v0 + 1, p1);
  if constexpr (NW == 4) {
    put(r2, e2, g2, cur + vw);
    load_2(v0 + 1, p2);
  }
  __syncthreads();
  f16v s, nx;
  float ref = 0.f;
  if (live) scores(nxt + kr + 32 * kKRow, qop, s);
  for (int v = v0; v < v1; ++v) {
    const int t0 = (v < ld.st.pre ? v : v + ld.st.shift) * kTok;
    __syncthreads();
    // (steps behind all of the wave's rows come last)
    if (live && t0 <= w.last) {
      const uint8_t *const k2 = cur + kr + 32 * kKRow, *const v2 = cur + vr + 32 * kVRow;
      if constexpr (NW == 4) {
        half_step<F32, M, 0, 4>(w, t0, h, qop, cur + kr, cur + vr, s, nx, o, m, ref, l, r1, e1, nxt + kw);
        half_step<F32, M, 0, 4>(w, t0 + 32, h, qop, k2, v2, nx, s, o, m, ref, l, r2, e2, nxt + vw);
      } else {
        half_step<F32, M, 0, 2>(w, t0, h, qop, cur + kr, cur + vr, s, nx, o, m, ref, l, r1, e1, nxt + w1);
        half_step<F32, M, 2, 2>(w, t0 + 32, h, qop, k2, v2, nx, s, o, m, ref, l, r1, e1, nxt + w1);
      }
    } else {
      store_block<M>(r1, (int)e1, nxt + w1);
      if constexpr (NW == 4) store_block<M>(r2, (int)e2, nxt + vw);
    }
    store_rest<M>(r1, e1, g1, nxt + w1);
    load_1(v + 2, n1);
    n1 = ld.page(v + 3, k1);
    if constexpr (NW == 4) {
      store_rest<M>(r2, e2, g2, nxt + vw);
      load_2(v + 2, n2);
      n2 = ld.page(v + 3, false);
    }
    uint8_t *const swap = cur;
    cur = nxt;
    nxt = swap;
  }
}

template <bool F32, int NW>
__global__ __launch_bounds__(64 * NW, 2)
void attn_tile_kernel(AttnPagedArgs a, int splits, int64_t tiles, int few_rows) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kStage];         // K and V of two steps
  constexpr int kRows = 32 * NW;
  const PageGeo &g = a.geo;
  const int t = threadIdx.x, lane = t & 63, h = lane >> 5, x = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  // KV heads run fastest, so that with eight of them an XCD reads one head's
  // pages; a sequence's last tiles, which see most tokens, come first
  const int Hkv = (int)g.Hkv, G = a.G;
  const uint32_t rest = blockIdx.x / (uint32_t)Hkv;
  const int kvh = (int)(blockIdx.x - rest * (uint32_t)Hkv);
  const int split = (int)(rest % (uint32_t)splits);
  int tile;
  Seq q;
  if (!find_tile<kRows>(a, rest / (uint32_t)splits, tiles, few_rows, q, tile)) return;
  const int64_t rows = (int64_t)q.n * G, r0 = (int64_t)tile * kRows;
  if (r0 >= rows || rows <= few_rows) return;
  const int64_t p0 = q.p0;
  const Steps st = steps_of<kTok>(a, q, p0 + r0 / G, p0 + (min(r0 + kRows, rows) - 1) / G);
  const int v0 = (int)((int64_t)st.count * split / splits);
  const int v1 = (int)((int64_t)st.count * (split + 1) / splits);

  // this lane's query row
  const int64_t wr = r0 + 32 * wave;
  const bool live = wr < rows;                             // of the wave
  const int64_t r = min(wr + x, rows - 1);
  const int tok = (int)(r / G), hd = kvh * G + (int)(r - (int64_t)tok * G);
  TileRow w;
  w.p = (int)(p0 + tok);
  w.pw0 = (int)(p0 + min(wr, rows - 1) / G);
  w.pw1 = (int)(p0 + (min(wr + 32, rows) - 1) / G);
  w.last = max(w.pw1, q.pre - 1);
  w.window = (int)(a.window && a.window < INT32_MAX ? a.window : INT32_MAX);
  w.pre = q.pre;
  w.sc = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * (a.softcap.cap > 0.f ? 1.f : kUnit<F32>);
  w.cap = a.softcap.cap;
  w.cap_k = a.softcap.k;
  w.biased = a.slopes != nullptr;
  w.slope = a.slopes ? a.slopes[hd] * kUnit<F32> : 0.f;

  // The score product's Q operand: 16 values of the reduction per product, lane half h
  // taking eight, in the slot order of their block.  A negative scale goes into its
  // sign; for a scale of zero Q is zero (a masked score, -inf, is scaled).
  bf8 qop[8];
  {
    const uint16_t *src = a.q + (int64_t)(q.row0 + tok) * a.q_ts + hd * a.q_hs;
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      u4 y = *(const u4 *)(src + 16 * ks + 8 * h);
      y = a.scale == 0.f ? u4{0u, 0u, 0u, 0u} : y ^ u4{sign, sign, sign, sign};
      if (split_slots(g.m[ks >> 1]))
        y = u4{__builtin_amdgcn_perm(y[1], y[0], 0x05040100), __builtin_amdgcn_perm(y[3], y[2], 0x05040100),
               __builtin_amdgcn_perm(y[1], y[0], 0x07060302), __builtin_amdgcn_perm(y[3], y[2], 0x07060302)};
      qop[ks] = __builtin_bit_cast(bf8, y);
    }
  }

  float m = -__builtin_inff(), l = 0.f;                    // l: this lane's tokens
  f16v o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  if (v0 < v1) {
    // (of eight waves, two on a SIMD: a wide block of K goes with a narrow one of V)
    const bool job_k = wave < 4;
    const int blk = job_k ? wave : 7 - wave;
    Loader ld;
    ld.pages = a.table + (int64_t)q.s * a.ld_table;
    ld.blk = blk;
    ld.plane = (int64_t)pick(g.off, blk) << g.lg_page;
    ld.page_rows = (uint32_t)Hkv << g.lg_page;
    ld.head_rows = (uint32_t)kvh << g.lg_page;
    ld.lane = lane;
    ld.last = q.len - 1;
    ld.lg_page = g.lg_page;
    ld.row = g.row;
    ld.n_pages = (int)g.pages;
    ld.st = st;
    ld.v1 = v1;
    const int bm = pick(g.m, blk);
    if (bm == 4) tile_steps<F32, NW, 4>(a, ld, v0, v1, job_k, live, w, qop, lds, o, m, l);
    else if (bm == 8) tile_steps<F32, NW, 8>(a, ld, v0, v1, job_k, live, w, qop, lds, o, m, l);
    else if (bm == 6) tile_steps<F32, NW, 6>(a, ld, v0, v1, job_k, live, w, qop, lds, o, m, l);
    else tile_steps<F32, NW, 3>(a, ld, v0, v1, job_k, live, w, qop, lds, o, m, l);
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

// o[row] = the splits' partial results merged in a fixed order.  GROUPS half waves
// take a row's splits in turn, eight at a time with their loads in flight together;
// their results are added pairwise.
constexpr int kMergeThreads = 256;
constexpr int kBatch = 8;
template <bool F32, int GROUPS>
__global__ __launch_bounds__(kMergeThreads)
void attn_merge_kernel(AttnPagedArgs a, int splits, int few_rows, int most, int64_t count) {
  constexpr int kRowsHere = kMergeThreads / 32 / GROUPS;
  __shared__ __attribute__((aligned(16))) float pos[GROUPS > 1 ? kMergeThreads / 32 : 1][kD];
  __shared__ float pms[kMergeThreads / 32], pls[kMergeThreads / 32];
  const int t = threadIdx.x, c = t & 31, grp = (t >> 5) % GROUPS, first = (t >> 5) - grp;
  const int64_t id = (int64_t)blockIdx.x * kRowsHere + (t >> 5) / GROUPS;
  bool here = id < count;                                  // (all meet at the barrier)
  int64_t row = here ? id : 0;
  if (!here) {
  } else if (most > 0) {                                   // row id % (most Hq) of a short sequence
    const int64_t per = most * a.Hq;
    const int s = (int)(id / per), c0 = a.cu_q[s], n = min(a.cu_q[s + 1] - c0, (int)a.max_q);
    const int64_t r = id - s * per;
    here = r < n * a.Hq && n * (int64_t)a.G <= few_rows && c0 >= 0 && c0 + (int64_t)n <= a.T;
    row = here ? c0 * a.Hq + r : 0;
  } else {
    const int tok = (int)(row / a.Hq), even = min(tok / (int)a.max_q, (int)a.S - 1);
    // its sequence: as if all had max_q rows, the loads in flight together (32 sequences of 40 rows:
    // 96.3 us, always searched 97.7), else the last one that begins at tok or before
    int c0 = a.cu_q[even], c1 = a.cu_q[even + 1];
    here = tok >= a.cu_q[0] && tok < a.cu_q[a.S];          // else no sequence's row
    if (here && (tok < c0 || tok >= c1)) {
      int lo = 0, hi = (int)a.S - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.cu_q[mid] <= tok) lo = mid;
        else hi = mid - 1;
      }
      c0 = a.cu_q[lo];
      c1 = a.cu_q[lo + 1];
    }
    const int n = min(c1 - c0, (int)a.max_q);              // not the other kernel's rows, nor those past max_q
    here = here && tok - c0 < n && (int64_t)n * a.G > few_rows;
  }
  if (!here) splits = 0;
  const float ninf = -__builtin_inff();
  float M = ninf, L = 0.f;
  f4 O = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = grp; s0 < splits; s0 += GROUPS * kBatch) {
    f2 ml[kBatch];
    f4 o[kBatch];
    float nm = M;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int s = min(s0 + GROUPS * u, splits - 1);
      ml[u] = *(const f2 *)part_ml(a, s, row);
      o[u] = *(const f4 *)(part_o(a, s, row) + 4 * c);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      // (a NaN sum has no maximum to go by, but counts; a split without a token has
      // no outputs)
      const bool none = s0 + GROUPS * u >= splits || (ml[u][0] == ninf && ml[u][1] == 0.f);
      if (none) ml[u] = f2{ninf, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) o[u][i] = none ? 0.f : o[u][i];
      nm = fmaxf(nm, ml[u][0]);
    }
    const float ref = nm == ninf ? 0.f : nm;
    const float f0 = weight<F32>(M - ref);
    L *= f0;
    O *= f0;
    M = nm;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float f = weight<F32>(ml[u][0] - ref);
      L += ml[u][0] == ninf ? ml[u][1] : ml[u][1] * f;
      O += o[u] * f;
    }
  }
  if constexpr (GROUPS > 1) {
    *(f4 *)(pos[t >> 5] + 4 * c) = O;
    if (c == 0) {
      pms[t >> 5] = M;
      pls[t >> 5] = L;
    }
  }
  if constexpr (GROUPS > 1) {
    __syncthreads();
    const float(*po)[kD] = pos + first, *pm = pms + first, *pl = pls + first;
    float Mx = ninf, Ls[GROUPS];
    f4 Os[GROUPS];
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) Mx = fmaxf(Mx, pm[k]);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const float f = pm[k] == ninf ? 1.f : weight<F32>(pm[k] - Mx);   // (without a score: 0 or a NaN)
      Ls[k] = pl[k] * f;
      Os[k] = *(const f4 *)(po[k] + 4 * c) * f;
    }
#pragma unroll
    for (int n = GROUPS / 2; n > 0; n /= 2)
#pragma unroll
      for (int k = 0; k < n; ++k) {
        Ls[k] += Ls[k + n];
        Os[k] += Os[k + n];
      }
    L = Ls[0];
    O = Os[0];
  }
  if (!here || grp > 0) return;
  O *= L == 0.f ? 0.f : 1.f / L;
  if (F32) *(f4 *)((float *)a.o + row * kD + 4 * c) = O;
  else *(bf4 *)((uint16_t *)a.o + row * kD + 4 * c) =
      bf4{(__bf16)O[0], (__bf16)O[1], (__bf16)O[2], (__bf16)O[3]};
}

// The rows of the tiles (most 0), or up to `most` rows of every short sequence.
void launch_merge(const AttnPagedArgs &a, int splits, int few_rows, int most, hipStream_t s) {
  const int64_t count = most > 0 ? a.S * most * a.Hq : a.T * a.Hq;
  // as many groups as the splits fill with one batch each (6880 rows of 9 splits: eight
  // groups 23.9 us, two 7)
  auto go = [&](auto fn, int groups) {
    hipLaunchKernelGGL(fn, dim3((unsigned)((count * groups + 7) / 8)), dim3(kMergeThreads), 0, s, a, splits,
                       few_rows, most, count);
  };
  if (splits <= kBatch) go(a.o_f32 ? attn_merge_kernel<true, 1> : attn_merge_kernel<false, 1>, 1);
  else if (splits <= 2 * kBatch) go(a.o_f32 ? attn_merge_kernel<true, 2> : attn_merge_kernel<false, 2>, 2);
  else go(a.o_f32 ? attn_merge_kernel<true, 8> : attn_merge_kernel<false, 8>, 8);
}

int64_t most_tiles(const AttnPagedArgs &a, int waves) { return a.T * a.G / (32 * waves) + a.S; }

// A dispatch holds fewer than 2^32 threads, and the tiles of many short sequences are
// launched whether they have rows or not: the splits that it has room for.
int64_t most_splits(const AttnPagedArgs &a, int waves) {
  const int64_t wgs = std::max<int64_t>(1, most_tiles(a, waves) * a.geo.Hkv);
  return std::max<int64_t>(1, UINT32_MAX / (64 * waves) / wgs);
}

// Which kernels run, and their splits (0: not launched).  Times in us, 64 query and 8
// KV heads, 4-bit cache, 256 CUs.
struct Plan {
  int tile, few;
  int waves;                             // of a tile
  int groups;                            // of 16 query rows, of the kernel for few
};
Plan plan_of(const AttnPagedArgs &a) {
  Plan p = {0, 0, 4, 1};
  const int64_t Hkv = a.geo.Hkv, most = a.max_q * a.G, cus = device_cu_count();
  const bool even = a.T == a.S * a.max_q;                  // every sequence has max_q tokens
  auto split = [](int64_t wgs, int64_t want, int64_t steps, int64_t least) {
    const int64_t n = std::min(want / std::max<int64_t>(wgs, 1), steps / least);
    return std::max<int64_t>(1, std::min<int64_t>(n, kMaxSplits));
  };
  if (most > kFewMost) {
    const int64_t steps = (a.max_kv + kTok - 1) / kTok;
    auto tiles = [&](int64_t rows) { return even ? a.S * ((most + rows - 1) / rows) : a.T * a.G / rows + 1; };
    // Splits: one round of workgroups (40 tokens of 4 sequences: 384 in 91, 864 in 107), of
    // at least four steps each (of max_kv tokens: a window is not looked at); a CU holds one
    // workgroup of eight waves, two of four.
    const int64_t t4 = tiles(128), t8 = tiles(256);
    const int64_t n4 = std::min(split(t4 * Hkv, 2 * cus, steps, 4), most_splits(a, 4));
    const int64_t n8 = std::min(split(t8 * Hkv, cus, steps, 4), most_splits(a, 8));
    // Eight waves share the dequantization of K and V among twice the query rows, but are
    // one workgroup per CU, whose start and end nothing covers.  They need whole rounds of
    // workgroups: new tokens over 16384, 2048 (two rounds) take 1036 against 1125 with four
    // waves, 480 (15 / 16 of one) 290 and 317, but 1536 (one and a half) 1011 and 930.  The
    // border is on the safe side of the crossing: 1664 (1.6 rounds) take 1012 and 1099, but
    // 2 prompts of 2731 in a window (2.7) 128 and 126.
    // They need tiles that are full: 112 tokens of 16 sequences, 896 rows of 1024, take 279
    // and 330, 40 of 4, 320 of 512, 82 and 80; safe again, 48 of 8, 384 of 512, take 87 and
    // 98, 80 of 32, 640 of 768, 410 and 436.
    // And rows that see the same steps, as those of a few tokens do: one query head per
    // KV head, 2 x 2048 tokens, 135 and 130.
    const int64_t wgs = t8 * Hkv * n8;
    const bool whole = 16 * wgs >= 15 * cus * ((wgs + cus - 1) / cus), full = 12 * t8 <= 7 * t4;
    p.waves = a.G >= 4 && whole && full ? 8 : 4;
    p.tile = (int)(p.waves == 8 ? n8 : n4);
  }
  // (in a mixed batch the two kernels share the sequences between them)
  if (!p.tile || (a.G <= kFewMost && !even)) {
    const int64_t chunks = (a.max_kv + kFewChunk - 1) / kFewChunk;
    // One round of workgroups; two where each keeps 1024 tokens, since the lengths of a
    // batch differ (32 sequences of 2048 to 8192 tokens: 61.6 and 52.9; 16 of 4096:
    // 23.6 and 25.2 with 512 tokens each).
    p.few = (int)std::max(split(a.S * Hkv, 2 * cus, chunks, 4), split(a.S * Hkv, 4 * cus, chunks, 32));
    p.groups = (p.tile ? a.G : most) <= 16 ? 1 : 2;
  }
  return p;
}

}  // namespace

int64_t attn_paged_work(const AttnPagedArgs &a) {
  const Plan p = plan_of(a);
  const int n = std::max(p.tile, p.few);
  const int64_t rows = n * a.T * a.Hq;
  return n <= 1 ? 0 : ((rows + 1) / 2 * 4 + rows * kD) * (int64_t)sizeof(float);
}

hipError_t launch_attn_paged(const AttnPagedArgs &args, hipStream_t s) {
  AttnPagedArgs a = args;
  const Plan p = plan_of(a);
  a.parts = std::max(p.tile, p.few);
  const int64_t tiles = most_tiles(a, p.waves);
  const int64_t wgs = tiles * a.geo.Hkv * p.tile;
  const int few_rows = p.few ? 16 * p.groups : 0;          // what the tiles leave to the other kernel
  const int most = (int)std::min<int64_t>(a.max_q, few_rows / a.G);
  if (p.few) {
    const hipError_t e = a.o_f32 ? launch_attn_few_f32(a, p.few, p.groups, s)
                                 : launch_attn_few_bf16(a, p.few, p.groups, s);
    if (e != hipSuccess) return e;
    if (p.few > 1) launch_merge(a, p.few, few_rows, most, s);
  }
  if (p.tile) {
    const auto fn = p.waves == 4 ? (a.o_f32 ? attn_tile_kernel<true, 4> : attn_tile_kernel<false, 4>)
                                 : (a.o_f32 ? attn_tile_kernel<true, 8> : attn_tile_kernel<false, 8>);
    hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3((unsigned)(64 * p.waves)), 0, s, a, p.tile, tiles,
                       few_rows);
    if (p.tile > 1) launch_merge(a, p.tile, few_rows, 0, s);
  }
  return hipGetLastError();
}

}  // namespace mxq
