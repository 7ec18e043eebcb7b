// api_paged.cpp -- the C ABI of rotary positions, the paged KV cache and the
// attention over it (declared in include/mxq.h): argument validation and kernel
// dispatch.  Every check happens before anything is enqueued; nothing here
// allocates, frees or synchronizes.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "../../include/mxq.h"
#include "mxq_device.h"
#include "mxq_internal.h"

namespace {

constexpr int64_t kD = 128;
constexpr int64_t kMaxGrid = (1 << 24) - 1;   // workgroups of 256: fewer than 2^32 threads

bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

mxq_status launched(hipError_t e) { return e == hipSuccess ? MXQ_OK : MXQ_ERR_DEVICE; }

mxq_status check_rotary(const mxq_rotary *r) {
  if (!r || !r->table) return MXQ_ERR_NULL;
  if (r->layout != MXQ_ROPE_HALVES && r->layout != MXQ_ROPE_PAIRS) return MXQ_ERR_UNSUPPORTED;
  if (r->rot < 2 || r->rot % 2 || r->rot > mxq::kRopeMaxRot) return MXQ_ERR_SHAPE;
  if (r->positions < 1 || r->positions > INT32_MAX) return MXQ_ERR_SHAPE;
  if (!aligned(r->table, 16)) return MXQ_ERR_ALIGN;
  return MXQ_OK;
}

mxq::RopeArgs rope_args(const mxq_rotary *r) {
  mxq::RopeArgs a{};
  if (r) {
    a.table = r->table;
    a.positions = r->positions;
    a.rot = r->rot;
    a.pairs = r->layout == MXQ_ROPE_PAIRS;
  }
  return a;
}

// The geometry of a page, from the format, the heads and the page's size.
mxq_status check_page(const mxq_fmt *fmt, int64_t Hkv, int32_t page, mxq::PageGeo *g) {
  mxq::Segs s;
  const mxq_status st = mxq::check_fmt(fmt, &s);
  if (st != MXQ_OK) return st;
  if (fmt->K != kD) return MXQ_ERR_SHAPE;
  if (fmt->perm) return MXQ_ERR_UNSUPPORTED;
  if (Hkv < 1 || Hkv > 65535) return MXQ_ERR_SHAPE;
  if (page < 16 || page > 1024 || (page & (page - 1))) return MXQ_ERR_SHAPE;
  *g = mxq::PageGeo{};
  int at = 0;
  for (int b = 0; b < 4; ++b) {
    g->m[b] = fmt->widths[b];
    g->off[b] = at;
    at += 4 * fmt->widths[b];
  }
  g->row = at;
  while ((1 << g->lg_page) < page) ++g->lg_page;
  g->Hkv = Hkv;
  return MXQ_OK;
}

mxq_status check_cache(const mxq_fmt *fmt, const mxq_paged_kv *c, mxq::PageGeo *g) {
  if (!c) return MXQ_ERR_NULL;
  const mxq_status st = check_page(fmt, c->Hkv, c->page_tokens, g);
  if (st != MXQ_OK) return st;
  if (c->reserved != 0) return MXQ_ERR_UNSUPPORTED;
  if (c->pages < 1 || c->pages > INT32_MAX || c->pages * c->page_tokens > INT32_MAX)
    return MXQ_ERR_SHAPE;
  if (!c->k_mant || !c->k_exp || !c->v_mant || !c->v_exp) return MXQ_ERR_NULL;
  if (!aligned(c->k_mant, 16) || !aligned(c->k_exp, 16) || !aligned(c->v_mant, 16) ||
      !aligned(c->v_exp, 16))
    return MXQ_ERR_ALIGN;
  g->pages = c->pages;
  return MXQ_OK;
}

// Strided rows whose heads hold 16-byte pieces.
mxq_status check_rows(const void *p, int64_t ts, int64_t hs) {
  if (!p) return MXQ_ERR_NULL;
  if (!aligned(p, 16) || ts % 8 || hs % 8) return MXQ_ERR_ALIGN;
  return MXQ_OK;
}

// Whether no two of T x H rows of D elements, ts and hs elements apart, overlap:
// nothing but i = j = 0 brings i ts + j hs, |i| < T, |j| < H, within D of zero.
bool rows_apart(int64_t T, int64_t ts, int64_t H, int64_t hs, int64_t D) {
  typedef __int128 wide;                                   // (of strides, and their multiples)
  const wide a = ts < 0 ? -(wide)ts : ts, b = hs < 0 ? -(wide)hs : hs;
  if ((T > 1 && a < D) || (H > 1 && b < D)) return false;
  if (T == 1 || H == 1) return true;
  if (a >= b ? a >= (H - 1) * b + D : b >= (T - 1) * a + D) return true;   // one within the other
  for (int64_t j = 1; j < H; ++j) {                        // the multiples of a around j b
    const wide i = j * b / a, over = j * b - i * a;
    if ((i < T && over < D) || (i + 1 < T && a - over < D)) return false;
  }
  return true;
}

mxq_status attn_shape(const mxq_fmt *fmt, const mxq_paged_kv *c, int64_t S, int64_t T, int64_t Hq,
                      int64_t max_q, int64_t max_kv, mxq::AttnPagedArgs *a) {
  const mxq_status st = check_cache(fmt, c, &a->geo);
  if (st != MXQ_OK) return st;
  if (S < 0 || T < 0 || max_q < 0 || max_kv < 0 || S > INT32_MAX - 1 || T > INT32_MAX ||
      max_q > INT32_MAX || max_kv > INT32_MAX)
    return MXQ_ERR_SHAPE;
  if (Hq < c->Hkv || Hq % c->Hkv || Hq / c->Hkv > 64) return MXQ_ERR_SHAPE;
  // (a dispatch holds fewer than 2^32 threads)
  if (T * Hq > (int64_t)1 << 29 || S * c->Hkv > (int64_t)1 << 22) return MXQ_ERR_SHAPE;
  a->S = S;
  a->T = T;
  a->Hq = Hq;
  a->G = (int)(Hq / c->Hkv);
  a->max_q = max_q < T ? max_q : T;
  a->max_kv = max_kv;
  return MXQ_OK;
}

}  // namespace

extern "C" {

mxq_status mxq_rope_table(const double *inv_freq, int32_t rot, int64_t positions, double mscale,
                          float *table, void *stream) {
  if (!inv_freq) return MXQ_ERR_NULL;
  const mxq_rotary r = {table, positions, rot, MXQ_ROPE_HALVES};
  const mxq_status st = check_rotary(&r);
  if (st != MXQ_OK) return st;
  if (!isfinite(mscale) || positions > kMaxGrid * 256 / (rot / 2)) return MXQ_ERR_SHAPE;
  for (int i = 0; i < rot / 2; ++i)
    if (!isfinite(inv_freq[i])) return MXQ_ERR_SHAPE;
  return launched(mxq::launch_rope_table(inv_freq, rot, positions, mscale, table,
                                         (hipStream_t)stream));
}

mxq_status mxq_rope(const mxq_rotary *rope, const uint16_t *x, int64_t T, int64_t H, int64_t D,
                    int64_t x_ts, int64_t x_hs, const int32_t *pos, uint16_t *y, int64_t y_ts,
                    int64_t y_hs, void *stream) {
  const mxq_status st = check_rotary(rope);
  if (st != MXQ_OK) return st;
  if (T < 0 || H < 0 || T > INT32_MAX || H > 65535 || D < rope->rot || D > 4096 || D % 2)
    return MXQ_ERR_SHAPE;
  if (T == 0 || H == 0) return MXQ_OK;
  if (!x || !y || !pos) return MXQ_ERR_NULL;
  if (!aligned(x, 4) || !aligned(y, 4) || x_ts % 2 || x_hs % 2 || y_ts % 2 || y_hs % 2)
    return MXQ_ERR_ALIGN;
  if (x == y && ((T > 1 && x_ts != y_ts) || (H > 1 && x_hs != y_hs))) return MXQ_ERR_SHAPE;
  if (T * H > kMaxGrid * 256 / (D / 2)) return MXQ_ERR_SHAPE;
  // rows of the result that overlap would be written, or turned in place, by several threads
  if (!rows_apart(T, y_ts, H, y_hs, D)) return MXQ_ERR_SHAPE;
  mxq::RopeRowsArgs a{};
  a.rope = rope_args(rope);
  a.x = x;
  a.y = y;
  a.pos = pos;
  a.T = T;
  a.H = H;
  a.D = D;
  a.x_ts = x_ts;
  a.x_hs = x_hs;
  a.y_ts = y_ts;
  a.y_hs = y_hs;
  return launched(mxq::launch_rope(a, (hipStream_t)stream));
}

int64_t mxq_kv_page_bytes(const mxq_fmt *fmt, int64_t Hkv, int32_t page_tokens) {
  mxq::PageGeo g;
  const mxq_status st = check_page(fmt, Hkv, page_tokens, &g);
  return st == MXQ_OK ? Hkv * page_tokens * g.row : -(int64_t)st;
}

int64_t mxq_kv_page_exp_bytes(const mxq_fmt *fmt, int64_t Hkv, int32_t page_tokens) {
  mxq::PageGeo g;
  const mxq_status st = check_page(fmt, Hkv, page_tokens, &g);
  return st == MXQ_OK ? Hkv * page_tokens * 4 : -(int64_t)st;
}

mxq_status mxq_kv_append(const mxq_fmt *fmt, const mxq_paged_kv *cache, const uint16_t *k,
                         int64_t k_ts, int64_t k_hs, const uint16_t *v, int64_t v_ts, int64_t v_hs,
                         int64_t T, const int64_t *slots, const int32_t *pos,
                         const mxq_rotary *rope, const uint16_t *q, int64_t Hq, int64_t q_ts,
                         int64_t q_hs, uint16_t *q_out, void *stream) {
  mxq::KvAppendArgs a{};
  mxq_status st = check_cache(fmt, cache, &a.geo);
  if (st != MXQ_OK) return st;
  if (rope) {
    st = check_rotary(rope);
    if (st != MXQ_OK) return st;
    if (rope->rot % 16 || rope->rot > kD) return MXQ_ERR_SHAPE;
  }
  if (T < 0 || T > INT32_MAX || Hq < 0 || Hq > 65535) return MXQ_ERR_SHAPE;
  if ((T + 15) / 16 * (2 * cache->Hkv + Hq) > kMaxGrid) return MXQ_ERR_SHAPE;
  if (T == 0) return MXQ_OK;
  if (!slots || (rope && !pos)) return MXQ_ERR_NULL;
  if ((st = check_rows(k, k_ts, k_hs)) != MXQ_OK) return st;
  if ((st = check_rows(v, v_ts, v_hs)) != MXQ_OK) return st;
  if (q) {
    if (Hq < 1) return MXQ_ERR_SHAPE;
    if ((st = check_rows(q, q_ts, q_hs)) != MXQ_OK) return st;
    if ((st = check_rows(q_out, 0, 0)) != MXQ_OK) return st;
    // (the stride of a single head or token is any)
    if (q == q_out && ((Hq > 1 && q_hs != kD) || (T > 1 && q_ts != Hq * kD))) return MXQ_ERR_SHAPE;
  }
  a.rope = rope_args(rope);
  a.k = k;
  a.v = v;
  a.k_ts = k_ts;
  a.k_hs = k_hs;
  a.v_ts = v_ts;
  a.v_hs = v_hs;
  if (q) {
    a.q = q;
    a.q_out = q_out;
    a.q_ts = q_ts;
    a.q_hs = q_hs;
    a.Hq = Hq;
  }
  a.T = T;
  a.slots = slots;
  a.pos = pos;
  a.k_mant = cache->k_mant;
  a.k_exp = cache->k_exp;
  a.v_mant = cache->v_mant;
  a.v_exp = cache->v_exp;
  a.ties_away = fmt->round == MXQ_ROUND_NEAREST_AWAY;
  a.full_clamp = fmt->clamp == MXQ_CLAMP_FULL;
  return launched(mxq::launch_kv_append(a, (hipStream_t)stream));
}

mxq_status mxq_kv_read(const mxq_fmt *fmt, const mxq_paged_kv *cache, const int64_t *slots,
                       int64_t n, uint16_t *k, uint16_t *v, void *stream) {
  mxq::KvReadArgs a{};
  const mxq_status st = check_cache(fmt, cache, &a.geo);
  if (st != MXQ_OK) return st;
  if (n < 0 || n > INT32_MAX || (n + 15) / 16 * 2 * cache->Hkv > kMaxGrid)
    return MXQ_ERR_SHAPE;
  if (n == 0 || (!k && !v)) return MXQ_OK;
  if (!slots) return MXQ_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16)) return MXQ_ERR_ALIGN;
  a.k_mant = cache->k_mant;
  a.k_exp = cache->k_exp;
  a.v_mant = cache->v_mant;
  a.v_exp = cache->v_exp;
  a.slots = slots;
  a.n = n;
  a.k = k;
  a.v = v;
  return launched(mxq::launch_kv_read(a, (hipStream_t)stream));
}

int64_t mxq_attn_paged_work_bytes(const mxq_fmt *fmt, const mxq_paged_kv *cache, int64_t S,
                                  int64_t T, int64_t Hq, int64_t max_q, int64_t max_kv) {
  mxq::AttnPagedArgs a{};
  const mxq_status st = attn_shape(fmt, cache, S, T, Hq, max_q, max_kv, &a);
  return st == MXQ_OK ? mxq::attn_paged_work(a) : -(int64_t)st;
}

mxq_status mxq_attn_paged(const mxq_fmt *fmt, const mxq_paged_kv *cache,
                          const mxq_paged_batch *batch, const mxq_attn_opts *opts,
                          const uint16_t *q, int64_t Hq, int64_t q_ts, int64_t q_hs, void *o,
                          int o_f32, float *work, int64_t work_bytes, void *stream) {
  if (!batch || !opts) return MXQ_ERR_NULL;
  mxq::AttnPagedArgs a{};
  mxq_status st = attn_shape(fmt, cache, batch->S, batch->T, Hq, batch->max_q, batch->max_kv, &a);
  if (st != MXQ_OK) return st;
  if (batch->table_pages < 0 || batch->table_pages > INT32_MAX ||
      (batch->S > 1 && batch->ld_table < batch->table_pages))
    return MXQ_ERR_SHAPE;
  if (!isfinite(opts->scale) || !isfinite(opts->softcap) || opts->softcap < 0.f ||
      (opts->softcap > 0.f && opts->softcap < 0x1p-60f) || opts->window < 0)
    return MXQ_ERR_SHAPE;
  if (a.S == 0 || a.T == 0 || a.max_q == 0) return MXQ_OK;
  if (!batch->cu_q || !batch->kv_len || (batch->table_pages > 0 && !batch->table) || !o)
    return MXQ_ERR_NULL;
  if ((st = check_rows(q, q_ts, q_hs)) != MXQ_OK) return st;
  if (!aligned(o, 16) || !aligned(work, 16)) return MXQ_ERR_ALIGN;
  const int64_t need = mxq::attn_paged_work(a);
  if (need > 0 && !work) return MXQ_ERR_NULL;
  if (work_bytes < need) return MXQ_ERR_SHAPE;
  a.k_mant = cache->k_mant;
  a.k_exp = cache->k_exp;
  a.v_mant = cache->v_mant;
  a.v_exp = cache->v_exp;
  a.q = q;
  a.q_ts = q_ts;
  a.q_hs = q_hs;
  a.o = o;
  a.o_f32 = o_f32 != 0;
  a.work = work;
  a.cu_q = batch->cu_q;
  a.kv_len = batch->kv_len;
  a.table = batch->table;
  a.ld_table = batch->ld_table;
  a.table_pages = batch->table_pages;
  a.prefix = opts->prefix;
  a.slopes = opts->slopes;
  a.window = opts->window;
  a.scale = opts->scale;
  const float cap = opts->softcap;
  if (cap > 0.f) a.softcap = {cap, (float)(2.0 * M_LOG2E / cap), -2.f * cap};
  return launched(mxq::launch_attn_paged(a, (hipStream_t)stream));
}

}  // extern "C"
