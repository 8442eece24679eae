// Host-side check of the operators of training in 8 bits of include/t5mi.h, as driver.cpp beside it (see
// tests/test_host_sanitizers_fp8.py).  Refusals and size queries over the range of every argument, and calls that pass the
// checks, for the arithmetic of their plans: every launch is turned away (T5_ERR_DEVICE), and pointers are never followed.
#include <climits>
#include <cmath>
#include <cstdio>
#include <vector>
#include "../../include/t5mi.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
  do {                                                                      \
    if (!(cond)) { std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)

static void* const P = (void*)4096;  // 256-byte aligned, never followed
static uint8_t* const S = (uint8_t*)P;

static void quantise() {
  const int64_t rows[] = {0, 1, 127, 128, 129, 70000, (1 << 24) + 1, ((int64_t)1 << 31) - 129}, cols[] = {1, 15, 16, 127, 128, 129, 5120, 1 << 23};
  for (int64_t r : rows)
    for (int64_t c : cols)
      for (int br : {1, 128})
        for (int ty : {T5_F32, T5_BF16})
          for (int q : {T5_E4M3, T5_E5M2}) {
            t5_quantize_cfg cfg = {r, c, c + 3, ty, q, br};
            const bool tiles = (r + 127) / 128 * ((c + 127) / 128) < (1 << 23), rows = br == 128 ? tiles : r * t5_fp8_scale_ld(c) < (1 << 29);
            EXPECT(t5_quantize_fp8(&cfg, P, P, S, nullptr, nullptr, nullptr) == (!rows ? T5_ERR_UNSUPPORTED : r ? T5_ERR_DEVICE : T5_OK));
            EXPECT(t5_quantize_fp8(&cfg, P, P, S, P, S, nullptr) == (!tiles ? T5_ERR_UNSUPPORTED : r ? T5_ERR_DEVICE : T5_OK));
            EXPECT(t5_fp8_ld(c) >= c && t5_fp8_ld(c) % 16 == 0 && t5_fp8_scale_ld(c) * 128 >= c && t5_fp8_scale_ld(c) % 4 == 0);
          }
  const t5_quantize_cfg bad[] = {{-1, 8, 8, 0, 2, 1}, {8, 0, 8, 0, 2, 1}, {8, 8, 7, 0, 2, 1}, {8, 8, 8, 2, 2, 1}, {8, 8, 8, 0, 1, 1}, {8, 8, 8, 0, 2, 2},
                                 {INT64_MAX, 8, 8, 0, 2, 1}, {8, INT64_MAX, INT64_MAX, 0, 2, 1}, {8, 8, INT64_MAX, 0, 2, 1}, {INT64_MIN, INT64_MIN, INT64_MIN, -1, -1, INT_MIN}};
  for (const auto& c : bad) EXPECT(t5_quantize_fp8(&c, P, P, S, P, S, nullptr) > T5_ERR_NULL);
}

static void product() {
  const int32_t ms[] = {0, 1, 32, 33, 64, 65, 255, 256, 257, 5000, 70000, 1 << 30}, ns[] = {1, 16, 255, 256, 5120, 131072, 1 << 30}, ks[] = {1, 128, 129, 5000, 65536, 1 << 23};
  for (int32_t m : ms)
    for (int32_t n : ns)
      for (int32_t k : ks)
        for (int f32 : {0, 1}) {
          const int64_t ld = t5_fp8_ld(k), ls = t5_fp8_scale_ld(k);
          t5_gemm_fp8_cfg c = {m, n, k, ld, ld, n, ls, ls, T5_E4M3 + f32, T5_E4M3, 1, 128, f32 ? T5_F32 : T5_BF16, f32};
          const size_t need = t5_gemm_fp8_workspace_bytes(&c);
          // (more than 2^31 tiles have no launch: an error of the device call too)
          EXPECT(t5_gemm_fp8(&c, P, S, P, S, P, need ? P : nullptr, need, nullptr) == (m ? T5_ERR_DEVICE : T5_OK));
          if (need) {
            EXPECT(t5_gemm_fp8(&c, P, S, P, S, P, P, need - 1, nullptr) == T5_ERR_WORKSPACE);
            EXPECT(t5_gemm_fp8(&c, P, S, P, S, P, S + 16, need, nullptr) == T5_ERR_WORKSPACE);
            EXPECT(need < ((size_t)1 << 29));
          }
        }
  const t5_gemm_fp8_cfg bad[] = {{INT_MIN, 1, 1, 16, 16, 1, 4, 4, 2, 2, 1, 1, 0, 0}, {1, INT_MAX, 1, 16, 16, INT_MAX, 4, 4, 2, 2, 1, 1, 0, 0},
                                 {1, 1, INT_MAX, INT64_MAX, INT64_MAX, 1, INT64_MAX, INT64_MAX, 2, 2, 1, 1, 0, 0}, {1, 1, 1, 16, 16, INT64_MAX, 4, 4, 2, 2, 1, 1, 0, 0},
                                 {1, 1, 1, INT64_MIN, 16, 1, 4, 4, 2, 2, 1, 1, 0, 0}};
  for (const auto& c : bad) EXPECT(t5_gemm_fp8(&c, P, S, P, S, P, P, (size_t)1 << 62, nullptr) > T5_ERR_NULL && t5_gemm_fp8_workspace_bytes(&c) == 0);
  EXPECT(t5_gemm_fp8_workspace_bytes(nullptr) == 0);
}

static void optimizer() {
  const adamw_cfg cfg = {1e-3, 0.9, 0.999, 1e-8, 1, 1, 2, nullptr};
  for (int n : {1, 39, 40, 41, 64, 65, 1000, 65536}) {
    std::vector<adamw_tensor> t(n);
    for (int i = 0; i < n; ++i)
      t[i] = {(float*)(uintptr_t)(((uintptr_t)(n - i) << 40) + 4096), P, P, P, S, S, i % 3 ? P : nullptr, i % 5 ? i + 1 : (int64_t)1 << 34, i % 2, i % 4 ? 8 : 32, 0.1};
    EXPECT(adamw_step_multi(t.data(), n, &cfg, nullptr) == T5_ERR_DEVICE);
    if (n > 1) {
      t[n - 1].param = t[n / 2].param + (n / 2 % 5 ? 0 : 5);
      EXPECT(adamw_step_multi(t.data(), n, &cfg, nullptr) == (n / 2 == n - 1 ? T5_ERR_DEVICE : T5_ERR_SHAPE));
    }
  }
  const adamw_cfg bad[] = {{-1, 0.9, 0.9, 1e-8, 1, 0, 0, nullptr}, {NAN, 0.9, 0.9, 1e-8, 1, 0, 0, nullptr}, {1, 1, 0.9, 1e-8, 1, 0, 0, nullptr}, {1, 0.9, -1, 1e-8, 1, 0, 0, nullptr},
                           {1, 0.9, 0.9, 0, 1, 0, 0, nullptr}, {1, 0.9, 0.9, 1e-8, 0, 0, 0, nullptr}, {1, 0.9, 0.9, 1e-8, INT_MIN, 0, 0, nullptr}};
  adamw_tensor t = {(float*)P, P, P, P, S, S, P, 10, 0, 8, 0};
  for (const auto& c : bad) EXPECT(adamw_step_multi(&t, 1, &c, nullptr) == T5_ERR_SHAPE);
  const adamw_cfg last = {1e-3, 0.9, 0.999, 1e-8, INT_MAX, UINT_MAX, UINT_MAX, nullptr};
  EXPECT(adamw_step_multi(&t, 1, &last, nullptr) == T5_ERR_DEVICE);
}

int main() {
  quantise();
  product();
  optimizer();
  std::printf("%s: %d failure(s)\n", failures ? "FAILED" : "OK", failures);
  return failures ? 1 : 0;
}
