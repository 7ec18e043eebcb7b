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

#include "attn_paged_device.h"

namespace mxq {

namespace {

constexpr int kTok = 64;                 // tokens per step
constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;       // query rows of a tile
constexpr int kFewMost = 32;             // query rows of the kernel for few
constexpr int kMaxSplits = 256;

// LDS rows of a token's 128 bf16 values: sixteen chunks of 16 bytes, chunk c of
// token t at c ^ swizzle(t).  Sixteen tokens' writes or operand reads of one chunk
// and a transposing read (four tokens, four adjacent chunks) lie in distinct banks.
constexpr int kTileBytes = kTok * kRowBytes;
__device__ inline int swizzle(int t) { return 4 * (t & 3) + ((t >> 2) & 3); }

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

template <bool F32>
__global__ __launch_bounds__(64 * kWaves, 2)
void attn_tile_kernel(AttnPagedArgs a, int splits, int64_t numbers, int few_rows) {
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
  if (r0 >= rows || rows <= few_rows) return;
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

// o[row] = the splits' partial results merged in a fixed order.  GROUPS half waves
// take a row's splits in turn, eight at a time with their loads in flight together;
// their results are added pairwise.
constexpr int kMergeThreads = 256;
constexpr int kBatch = 8;
template <bool F32, int GROUPS>
__global__ __launch_bounds__(kMergeThreads)
void attn_merge_kernel(AttnPagedArgs a, int tile, int few, int few_rows) {
  constexpr int kRowsHere = kMergeThreads / 32 / GROUPS;
  __shared__ __attribute__((aligned(16))) float po[GROUPS > 1 ? GROUPS : 1][kD];
  __shared__ float pm[GROUPS], pl[GROUPS];
  const int t = threadIdx.x, c = t & 31, grp = (t >> 5) % GROUPS;
  const int64_t row = (int64_t)blockIdx.x * kRowsHere + (t >> 5) / GROUPS;
  if (row >= a.T * a.Hq) return;                           // (uniform where the groups meet)
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
    if ((int64_t)(a.cu_q[lo + 1] - a.cu_q[lo]) * a.G <= few_rows) splits = few;
    if (splits == 1) return;                               // written already
  }
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
    *(f4 *)(po[grp] + 4 * c) = O;
    if (c == 0) {
      pm[grp] = M;
      pl[grp] = L;
    }
    __syncthreads();
    if (grp > 0) return;
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
  O *= L == 0.f ? 0.f : 1.f / L;
  if (F32) *(f4 *)((float *)a.o + row * kD + 4 * c) = O;
  else *(bf4 *)((uint16_t *)a.o + row * kD + 4 * c) =
      bf4{(__bf16)O[0], (__bf16)O[1], (__bf16)O[2], (__bf16)O[3]};
}

template <bool F32>
void launch_merge(const AttnPagedArgs &a, int tile, int few, int few_rows, hipStream_t s) {
  const int64_t rows = a.T * a.Hq;
  if (std::max(tile, few) <= kBatch)
    hipLaunchKernelGGL((attn_merge_kernel<F32, 1>), dim3((unsigned)((rows + 7) / 8)),
                       dim3(kMergeThreads), 0, s, a, tile, few, few_rows);
  else
    hipLaunchKernelGGL((attn_merge_kernel<F32, 8>), dim3((unsigned)rows), dim3(kMergeThreads), 0, s,
                       a, tile, few, few_rows);
}

int64_t tile_numbers(const AttnPagedArgs &a) { return a.T * a.G / kRows + a.S; }

// Splits of each kernel (0 where it is not launched), and the groups of 16 query
// rows that the kernel for few rows takes.
struct Plan {
  int tile, few, groups;
};
Plan plan_of(const AttnPagedArgs &a) {
  Plan p = {0, 0, 1};
  const int64_t Hkv = a.geo.Hkv, most = a.max_q * a.G;
  auto split = [](int64_t wgs, int64_t want, int64_t steps, int64_t least) {
    const int64_t n = std::min(want / std::max<int64_t>(wgs, 1), steps / least);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, kMaxSplits));
  };
  if (most > kFewMost) p.tile = split(tile_numbers(a) * Hkv, 1024, (a.max_kv + kTok - 1) / kTok, 4);
  // (every sequence has max_q rows where their sum says so)
  if (!p.tile || (a.G <= kFewMost && a.T < a.S * a.max_q)) {
    p.few = split(a.S * Hkv, 512, (a.max_kv + kFewChunk - 1) / kFewChunk, 4);
    p.groups = (p.tile ? a.G : most) <= 16 ? 1 : 2;
  }
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
  const int64_t wgs = numbers * a.geo.Hkv * p.tile;
  const int few_rows = p.few ? 16 * p.groups : 0;          // what the tiles leave to the other kernel
  // (a dispatch holds fewer than 2^32 threads)
  if (std::max({wgs, a.S * a.geo.Hkv * p.few, a.parts > 1 ? a.T * a.Hq : 0}) >= ((int64_t)1 << 32) / 256)
    return hipErrorInvalidValue;
  hipError_t e = hipSuccess;
  if (p.few) {
    e = a.o_f32 ? launch_attn_few_f32(a, p.few, p.groups, s) : launch_attn_few_bf16(a, p.few, p.groups, s);
    if (e != hipSuccess) return e;
  }
  if (p.tile) {
    const auto fn = a.o_f32 ? attn_tile_kernel<true> : attn_tile_kernel<false>;
    hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(64 * kWaves), 0, s, a, p.tile, numbers, few_rows);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.parts <= 1) return e;
  const int tile = p.tile ? p.tile : p.few, few = p.few ? p.few : p.tile;
  if (a.o_f32) launch_merge<true>(a, tile, few, few_rows, s);
  else launch_merge<false>(a, tile, few, few_rows, s);
  return hipGetLastError();
}

}  // namespace mxq
