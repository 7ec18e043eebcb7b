// api_experts.cpp -- the C ABI of routing, plans and the weighted sum of experts
// (declared in include/mxq.h): argument validation and kernel dispatch.  Every
// check happens before anything is enqueued; nothing here allocates, frees or
// synchronizes.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "../../include/mxq.h"
#include "mxq_internal.h"

namespace {

constexpr int64_t kMaxPairs = (int64_t)1 << 26;
constexpr int64_t kMaxGrid = (1 << 24) - 1;   // workgroups of 256: fewer than 2^32 threads

bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

mxq_status launched(hipError_t e) { return e == hipSuccess ? MXQ_OK : MXQ_ERR_DEVICE; }

mxq_status check_counts(int64_t pairs, int64_t experts) {
  return pairs < 0 || pairs > kMaxPairs || experts < 1 || experts > mxq::kMaxExperts ? MXQ_ERR_SHAPE
                                                                                     : MXQ_OK;
}

int64_t expert_rows(int64_t pairs, int64_t experts) {
  return (pairs + 15 * (pairs < experts ? pairs : experts)) & ~(int64_t)15;
}

mxq_status check_work(const mxq_experts *p) {
  if (!p->work) return MXQ_ERR_NULL;
  return aligned(p->work, 16) ? MXQ_OK : MXQ_ERR_ALIGN;
}

mxq::PlanArgs plan_args(const mxq::Groups &g, const int32_t *ids, int32_t *work) {
  mxq::PlanArgs a{};
  a.work = work;
  a.ids = ids;
  a.pairs = g.pairs;
  a.rows = g.rows;
  a.E = g.E;
  a.first = const_cast<int32_t *>(g.first);
  a.pair = const_cast<int32_t *>(g.pair);
  return a;
}

}  // namespace

namespace mxq {

mxq_status check_experts(const mxq_experts *p, Groups *g) {
  if (!p) return MXQ_ERR_NULL;
  if (p->reserved != 0) return MXQ_ERR_UNSUPPORTED;
  const mxq_status st = check_counts(p->pairs, p->experts);
  if (st != MXQ_OK) return st;
  if (!p->first || (p->pairs > 0 && !p->pair)) return MXQ_ERR_NULL;
  if (!aligned(p->first, 16) || !aligned(p->pair, 16)) return MXQ_ERR_ALIGN;
  *g = Groups{};
  g->first = p->first;
  g->pair = p->pair;
  g->E = p->experts;
  g->rows = expert_rows(p->pairs, p->experts);
  g->pairs = p->pairs;
  return MXQ_OK;
}

}  // namespace mxq

extern "C" {

int64_t mxq_expert_rows(int64_t pairs, int32_t experts) {
  const mxq_status st = check_counts(pairs, experts);
  return st == MXQ_OK ? expert_rows(pairs, experts) : -(int64_t)st;
}

mxq_status mxq_expert_plan(const int32_t *ids, const mxq_experts *plan, void *stream) {
  mxq::Groups g;
  mxq_status st = mxq::check_experts(plan, &g);
  if (st != MXQ_OK || (st = check_work(plan)) != MXQ_OK) return st;
  if (g.pairs > 0 && !ids) return MXQ_ERR_NULL;
  if (!aligned(ids, 16)) return MXQ_ERR_ALIGN;
  return launched(mxq::launch_expert_plan(plan_args(g, ids, plan->work), (hipStream_t)stream));
}

mxq_status mxq_route(const mxq_route_opts *opts, const void *logits, int logits_f32, int64_t T,
                     int64_t ld, int32_t *ids, float *weights, const mxq_experts *plan,
                     void *stream) {
  if (!opts) return MXQ_ERR_NULL;
  mxq::Groups g;
  mxq_status st = mxq::check_experts(plan, &g);
  if (st != MXQ_OK || (st = check_work(plan)) != MXQ_OK) return st;
  if (opts->score != MXQ_SCORE_SOFTMAX && opts->score != MXQ_SCORE_SIGMOID)
    return MXQ_ERR_UNSUPPORTED;
  if (opts->k < 1 || opts->k > 32 || opts->k > g.E || !isfinite(opts->scale)) return MXQ_ERR_SHAPE;
  if (T < 0 || T > kMaxGrid * 4 || T * opts->k != g.pairs || (T > 1 && ld < g.E)) return MXQ_ERR_SHAPE;
  if (T > 0 && (!logits || !ids || !weights)) return MXQ_ERR_NULL;
  if (!aligned(logits, logits_f32 ? 4 : 2) || !aligned(ids, 16) || !aligned(weights, 16) ||
      !aligned(opts->bias, 4))
    return MXQ_ERR_ALIGN;
  mxq::RouteArgs a{};
  a.logits = logits;
  a.logits_f32 = logits_f32 != 0;
  a.T = T;
  a.ld = ld;
  a.E = g.E;
  a.k = opts->k;
  a.score = opts->score;
  a.normalise = opts->normalise != 0;
  a.scale = opts->scale;
  a.bias = opts->bias;
  a.ids = ids;
  a.weights = weights;
  return launched(mxq::launch_route(a, plan_args(g, ids, plan->work), (hipStream_t)stream));
}

static mxq_status quantize_experts(const mxq_fmt *fmt, const mxq_experts *plan,
                                   const int32_t *perms, const uint16_t *src, const uint16_t *src2,
                                   int64_t per_row, int64_t ld, uint8_t *mant, uint8_t *exp,
                                   void *stream) {
  mxq::Groups g;
  const mxq_status st = mxq::check_experts(plan, &g);
  if (st != MXQ_OK) return st;
  if (per_row < 1 || per_row > INT32_MAX || g.pairs % per_row) return MXQ_ERR_SHAPE;
  if (!aligned(perms, 16)) return MXQ_ERR_ALIGN;
  return mxq::quantize_common(fmt, src, g.pairs / per_row, ld, mant, exp, stream, mxq::kImage, nullptr, 0.f,
                         src2, &g, per_row, perms);
}

mxq_status mxq_quantize_act_experts(const mxq_fmt *fmt, const mxq_experts *plan,
                                    const int32_t *perms, const uint16_t *a, int64_t per_row,
                                    int64_t lda, uint8_t *a_mant, uint8_t *a_exp, void *stream) {
  return quantize_experts(fmt, plan, perms, a, nullptr, per_row, lda, a_mant, a_exp, stream);
}

mxq_status mxq_quantize_act_swiglu_experts(const mxq_fmt *fmt, const mxq_experts *plan,
                                           const int32_t *perms, const uint16_t *gate,
                                           const uint16_t *up, int64_t per_row, int64_t ld,
                                           uint8_t *a_mant, uint8_t *a_exp, void *stream) {
  if (plan && plan->pairs > 0 && !up) return MXQ_ERR_NULL;
  return quantize_experts(fmt, plan, perms, gate, up, per_row, ld, a_mant, a_exp, stream);
}

mxq_status mxq_gemm_experts(const mxq_fmt *fmt, const mxq_experts *plan, int64_t N,
                            const uint8_t *a_mant, const uint8_t *a_exp, const uint8_t *w_mant,
                            const uint8_t *w_exp, void *y, int y_f32, int64_t ldy, void *stream) {
  mxq::Groups x;
  mxq_status st = mxq::check_experts(plan, &x);
  if (st != MXQ_OK) return st;
  mxq::GemmArgs g;
  st = mxq::gemm_args(fmt, x.pairs, N, a_mant, a_exp, w_mant, w_exp, y, &g);
  if (st != MXQ_OK) return st;
  if (x.pairs == 0 || N == 0) return MXQ_OK;
  if (ldy < N || N > INT32_MAX) return MXQ_ERR_SHAPE;
  g.x = x;
  g.w_expert = mxq_weight_bytes(fmt, N);
  g.w_expert_sc = mxq_weight_exp_bytes(fmt, N);
  g.y = (float *)y;
  g.y_bf16 = !y_f32;
  g.ldy = ldy;
  if (mxq::gemm_experts_workgroups(g) > kMaxGrid) return MXQ_ERR_SHAPE;
  return launched(mxq::launch_gemm_experts(g, (hipStream_t)stream));
}

mxq_status mxq_combine_experts(const void *y, int y_f32, int64_t ldy, const int32_t *ids,
                               const float *weights, int64_t T, int64_t k, int32_t experts,
                               int64_t N, const uint16_t *residual, int64_t ldr, void *out,
                               int out_f32, int64_t ldo, void *stream) {
  if (T < 0 || N < 0 || k < 1 || experts < 1 || T > kMaxPairs || k > kMaxPairs || T * k > kMaxPairs)
    return MXQ_ERR_SHAPE;
  if (N > INT32_MAX || ldy < N || ldo < N || (residual && ldr < N)) return MXQ_ERR_SHAPE;
  if (T == 0 || N == 0) return MXQ_OK;
  if (!y || !ids || !weights || !out) return MXQ_ERR_NULL;
  if (!aligned(y, y_f32 ? 4 : 2) || !aligned(out, out_f32 ? 4 : 2) || !aligned(ids, 4) ||
      !aligned(weights, 4) || !aligned(residual, 2))
    return MXQ_ERR_ALIGN;
  // (in place, a thread reads what it writes)
  if (residual == out && (out_f32 || (T > 1 && ldr != ldo))) return MXQ_ERR_SHAPE;
  mxq::CombineArgs a{};
  a.y = y;
  a.y_f32 = y_f32 != 0;
  a.out_f32 = out_f32 != 0;
  a.ldy = ldy;
  a.T = T;
  a.k = k;
  a.N = N;
  a.ldr = ldr;
  a.ldo = ldo;
  a.E = experts;
  a.ids = ids;
  a.weights = weights;
  a.residual = residual;
  a.out = out;
  return launched(mxq::launch_combine(a, (hipStream_t)stream));
}

}  // extern "C"
