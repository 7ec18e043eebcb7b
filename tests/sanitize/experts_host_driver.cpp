// Host-side driver of the entry points of layers with experts, and of norms of
// queries and keys, for the sanitizer build (test infrastructure).  Built host-only
// with AddressSanitizer and UndefinedBehaviorSanitizer and run on a machine without a
// GPU: size queries and argument checks run for real; calls that pass them reach a
// kernel launch, which the HIP runtime refuses without a device, so they must return
// MXQ_ERR_DEVICE.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <vector>

#include "../../include/mxq.h"

static int failures = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      fprintf(stderr, "%s:%d: expectation failed: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                          \
    }                                                                      \
  } while (0)

int main() {
  // a large, aligned, never dereferenced address stands in for device memory
  void *fake = (void *)(uintptr_t)(1u << 20);
  uint16_t *f16 = (uint16_t *)fake;
  uint8_t *f8 = (uint8_t *)fake;
  float *f32 = (float *)fake;
  int32_t *i32 = (int32_t *)fake;
  const int64_t *i64 = (const int64_t *)fake;
  for (int64_t pairs : std::vector<int64_t>{0, 1, 17, 4096, 1 << 26, (1 << 26) + 1, -1, INT64_MAX, INT64_MIN})
    for (int32_t E : {1, 7, 128, 1024, 1025, 0, -1, INT32_MIN, INT32_MAX}) {
      const int64_t rows = mxq_expert_rows(pairs, E);
      const bool good = pairs >= 0 && pairs <= 1LL << 26 && E >= 1 && E <= 1024;
      EXPECT(good ? rows >= pairs && rows % 16 == 0 : rows < 0);
    }
  const std::vector<std::vector<uint8_t>> maps = {
      {4}, {3}, {6}, {8}, {3, 4, 6, 8}, {4, 4, 4, 4, 4, 6, 8}, std::vector<uint8_t>(448, 4)};
  for (const auto &w : maps)
    for (int clamp = 0; clamp < 2; ++clamp) {
      const int64_t K = 32 * (int64_t)w.size();
      const mxq_fmt f = {K, 32, 0, clamp, 0, w.data(), nullptr};
      for (int64_t T : {1, 5, 33, 300, 5000})
        for (int32_t k : {1, 2, 8})
          for (int32_t E : {8, 100, 1024}) {
            const mxq_experts p = {T * k, E, 0, i32, i32, i32};
            for (int score = 0; score < 2; ++score) {
              const mxq_route_opts o = {k, score, 1, 1.f, score ? f32 : nullptr};
              EXPECT(mxq_route(&o, fake, score, T, E, i32, f32, &p, nullptr) == MXQ_ERR_DEVICE);
            }
            EXPECT(mxq_expert_plan(i32, &p, nullptr) == MXQ_ERR_DEVICE);
            for (const int32_t *perms : {(const int32_t *)nullptr, (const int32_t *)i32}) {
              EXPECT(mxq_quantize_act_experts(&f, &p, perms, f16, k, K + 3, f8, f8, nullptr) ==
                     MXQ_ERR_DEVICE);
              EXPECT(mxq_quantize_act_swiglu_experts(&f, &p, perms, f16, f16, 1, 2 * K, f8, f8, nullptr) ==
                     MXQ_ERR_DEVICE);
            }
            for (int64_t N : {1, 130, 28672})
              for (int y32 = 0; y32 < 2; ++y32)
                EXPECT(mxq_gemm_experts(&f, &p, N, f8, f8, f8, f8, fake, y32, N + 5, nullptr) ==
                       MXQ_ERR_DEVICE);
          }
    }
  // sizes at their limits
  {
    const uint8_t w[1] = {4};
    const mxq_fmt f = {32, 32, 0, 0, 0, w, nullptr};
    const mxq_experts p = {1LL << 26, 1024, 0, i32, i32, i32};
    EXPECT(mxq_expert_plan(i32, &p, nullptr) == MXQ_ERR_DEVICE);
    EXPECT(mxq_gemm_experts(&f, &p, 128, f8, f8, f8, f8, fake, 1, 128, nullptr) == MXQ_ERR_DEVICE);
    EXPECT(mxq_gemm_experts(&f, &p, INT32_MAX, f8, f8, f8, f8, fake, 1, INT64_MAX, nullptr) ==
           MXQ_ERR_SHAPE);
    const mxq_route_opts o = {1, 0, 0, 1.f, nullptr};
    EXPECT(mxq_route(&o, fake, 1, 1LL << 26, 1024, i32, f32, &p, nullptr) == MXQ_ERR_SHAPE);
    for (int64_t N : std::vector<int64_t>{1, 4096, (int64_t)1 << 31, INT64_MAX})
      for (int64_t T : std::vector<int64_t>{1, 1 << 20, 1 << 26, INT64_MAX}) {
        const int s = mxq_combine_experts(fake, 0, N, i32, f32, T, 1, 8, N, f16, N, f32 + 64, 0, N, nullptr);
        EXPECT(s == MXQ_ERR_SHAPE || s == MXQ_ERR_DEVICE);
      }
  }
  for (int64_t k : {1, 6, 32})
    for (int64_t N : {1, 33, 4096})
      EXPECT(mxq_combine_experts(fake, 1, N + 3, i32, f32, 70, k, 8, N, nullptr, 0, f32, 1, N, nullptr) ==
             MXQ_ERR_DEVICE);
  // norms of queries and keys
  const mxq_qk_norm n = {f16, f16, 1e-6f};
  for (int64_t D : {2, 66, 128, 520, 4096})
    for (int layout = 0; layout < 2; ++layout) {
      const mxq_rotary r = {f32, 4096, (int32_t)(D < 512 ? D : 512), layout};
      for (int64_t T : {1, 4001})
        EXPECT(mxq_rope_qk(&r, &n, i32, T, D, f16, 5, 5 * D, D, f16 + 64, 5 * D, D, f16, 2, 2 * D, D, f16 + 128,
                           2 * D, D, nullptr) == MXQ_ERR_DEVICE);
      EXPECT(mxq_rope_qk(&r, &n, i32, INT32_MAX, D, f16, 65535, INT64_MAX - 1, D, f16 + 64, INT64_MAX - 1, D,
                         nullptr, 0, 0, 0, nullptr, 0, 0, nullptr) == MXQ_ERR_SHAPE);
    }
  const uint8_t w4[4] = {3, 4, 6, 8};
  const mxq_fmt f = {128, 32, 0, 0, 0, w4, nullptr};
  const mxq_paged_kv kv = {100, 8, 64, 0, f8, f8, f8, f8};
  const mxq_rotary r = {f32, 4096, 128, MXQ_ROPE_PAIRS};
  EXPECT(mxq_kv_append_norm(&f, &kv, &n, f16, 1024, 128, f16, 1024, 128, 33, i64, i32, &r, f16, 64, 8192, 128,
                            f16, nullptr) == MXQ_ERR_DEVICE);
  if (failures) return 1;
  printf("experts host driver: ok\n");
  return 0;
}
