// Host-side driver of the rotary, paged-cache and paged-attention entry points
// for the sanitizer build (test infrastructure).  Built host-only with
// AddressSanitizer and UndefinedBehaviorSanitizer and run on a machine without a
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
  const int32_t *i32 = (const int32_t *)fake;
  const int64_t *i64 = (const int64_t *)fake;
  const uint8_t set[4] = {3, 4, 6, 8};
  for (int a = 0; a < 4; ++a)
    for (int b = a; b < 4; ++b)
      for (int c = b; c < 4; ++c)
        for (int d = c; d < 4; ++d) {
          const uint8_t w[4] = {set[a], set[b], set[c], set[d]};
          mxq_fmt f = {128, 32, 0, 0, 0, w, nullptr};
          for (int page = 16; page <= 1024; page *= 2) {
            EXPECT(mxq_kv_page_bytes(&f, 8, page) == 8LL * page * 4 * (w[0] + w[1] + w[2] + w[3]));
            EXPECT(mxq_kv_page_exp_bytes(&f, 8, page) == 8LL * page * 4);
          }
          mxq_paged_kv kv = {100, 8, 64, 0, f8, f8, f8, f8};
          const mxq_rotary r = {f32, 4096, 128, MXQ_ROPE_PAIRS};
          EXPECT(mxq_kv_append(&f, &kv, f16, 1024, 128, f16, 1024, 128, 33, i64, i32, &r, f16, 64, 8192, 128,
                               f16, nullptr) == MXQ_ERR_DEVICE);
          EXPECT(mxq_kv_append(&f, &kv, f16, 1024, 128, f16, 1024, 128, 1, i64, nullptr, nullptr, nullptr, 0,
                               0, 0, nullptr, nullptr) == MXQ_ERR_DEVICE);
          EXPECT(mxq_kv_read(&f, &kv, i64, 5, f16, nullptr, nullptr) == MXQ_ERR_DEVICE);
          for (int64_t S : {1, 3, 70})
            for (int64_t q : {1, 5, 300, 5000})
              for (int64_t len : {0, 1, 4000, 1 << 20})
                for (int64_t Hq : {8, 40, 64, 256, 512}) {
                  const int64_t T = S * q - (S > 1 ? 1 : 0);
                  const int64_t need = mxq_attn_paged_work_bytes(&f, &kv, S, T, Hq, q, len);
                  EXPECT(need >= 0 && need % 16 == 0);
                  const mxq_paged_batch bt = {S, T, q, len, i32, i32, i32, 40, 40};
                  const mxq_attn_opts o = {0.1f, 30.f, 128, i32, f32};
                  for (int fp32 = 0; fp32 < 2; ++fp32)
                    EXPECT(mxq_attn_paged(&f, &kv, &bt, &o, f16, Hq, Hq * 128, 128, fake, fp32, f32, need,
                                          nullptr) == MXQ_ERR_DEVICE);
                  if (need > 0)
                    EXPECT(mxq_attn_paged(&f, &kv, &bt, &o, f16, Hq, Hq * 128, 128, fake, 0, f32, need - 1,
                                          nullptr) == MXQ_ERR_SHAPE);
                }
        }
  const uint8_t w4[4] = {4, 4, 4, 4};
  mxq_fmt f = {128, 32, 0, 0, 0, w4, nullptr};
  // the ends of the ranges: no overflow on the way to a refusal
  for (int64_t big : {(int64_t)INT32_MAX, (int64_t)INT32_MAX + 1, INT64_MAX, INT64_MIN, (int64_t)-1}) {
    mxq_paged_kv kv = {big, 8, 64, 0, f8, f8, f8, f8};
    EXPECT(mxq_kv_read(&f, &kv, i64, 5, f16, f16, nullptr) == MXQ_ERR_SHAPE);
    kv = {100, big, 64, 0, f8, f8, f8, f8};
    EXPECT(mxq_kv_read(&f, &kv, i64, 5, f16, f16, nullptr) == MXQ_ERR_SHAPE);
    kv = {100, 8, 64, 0, f8, f8, f8, f8};
    EXPECT(mxq_kv_read(&f, &kv, i64, big, f16, f16, nullptr) == MXQ_ERR_SHAPE);
    EXPECT(mxq_kv_append(&f, &kv, f16, 1024, 128, f16, 1024, 128, big, i64, i32, nullptr, f16, 64, 8192, 128,
                         f16, nullptr) == MXQ_ERR_SHAPE);
    EXPECT(mxq_kv_append(&f, &kv, f16, 1024, 128, f16, 1024, 128, 7, i64, i32, nullptr, f16, big, 8192, 128,
                         f16, nullptr) == MXQ_ERR_SHAPE);
    EXPECT(mxq_attn_paged_work_bytes(&f, &kv, big, 4, 8, 4, 4) < 0);
    EXPECT(mxq_attn_paged_work_bytes(&f, &kv, 4, big, 8, 4, 4) < 0);
    EXPECT(mxq_attn_paged_work_bytes(&f, &kv, 4, 4, big, 4, 4) < 0);
    const mxq_rotary r = {f32, 4096, 128, MXQ_ROPE_HALVES};
    EXPECT(mxq_rope(&r, f16, big, 8, 128, 1024, 128, i32, f16, 1024, 128, nullptr) == MXQ_ERR_SHAPE);
    EXPECT(mxq_rope(&r, f16, 8, big, 128, 1024, 128, i32, f16, 1024, 128, nullptr) == MXQ_ERR_SHAPE);
    EXPECT(mxq_rope(&r, f16, 8, 8, big, 1024, 128, i32, f16, 1024, 128, nullptr) == MXQ_ERR_SHAPE);
  }
  mxq_paged_kv kv = {100, 8, 64, 0, f8, f8, f8, f8};
  EXPECT(mxq_attn_paged_work_bytes(&f, &kv, 4, 4, 8, INT32_MAX, INT32_MAX) >= 0);
  EXPECT(mxq_attn_paged_work_bytes(&f, &kv, 1 << 19, 1 << 19, 8, 1, INT32_MAX) >= 0);
  std::vector<double> freq(256, 0.5);
  EXPECT(mxq_rope_table(freq.data(), 512, 100, 1.0, f32, nullptr) == MXQ_ERR_DEVICE);
  freq.resize(1);
  EXPECT(mxq_rope_table(freq.data(), 2, 100, 1.0, f32, nullptr) == MXQ_ERR_DEVICE);
  for (int layout = 0; layout < 2; ++layout)
    for (int rot : {2, 20, 64, 128}) {
      const mxq_rotary r = {f32, 4096, rot, layout};
      EXPECT(mxq_rope(&r, f16, 9, 3, 128, 384, 128, i32, f16, 384, 128, nullptr) == MXQ_ERR_DEVICE);
      EXPECT(mxq_rope(&r, f16, 9, 3, 130, 390, 130, i32, f16, 390, 130, nullptr) == MXQ_ERR_DEVICE);
    }
  if (failures) return 1;
  printf("paged host driver: ok\n");
  return 0;
}
