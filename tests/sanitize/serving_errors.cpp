// Host-side argument checks of the calls around a decoding step under AddressSanitizer and
// UndefinedBehaviorSanitizer (built by tests/test_serving_sanitize.py with the library's host code
// instrumented). Every call is refused on the host before anything is enqueued; pointers are fake
// device addresses that are never dereferenced. Each size argument takes the extremes of its type in
// turn, where a product of sizes in a check could overflow.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "hsa_step.h"

static int failures = 0;
static void refused(int got, const char* what, long long value) {
  if (got == HSA_STEP_OK || got == HSA_STEP_ERR_LAUNCH) {
    fprintf(stderr, "%s = %lld: returned %d\n", what, value, got);
    ++failures;
  }
}

static void* P(int i) { return reinterpret_cast<void*>(0x100000000000ull + 0x10000000000ull * i); }
static int32_t* I(int i) { return static_cast<int32_t*>(P(i)); }
static int8_t* B(int i) { return static_cast<int8_t*>(P(i)); }
static float* F(int i) { return static_cast<float*>(P(i)); }

int main() {
  const int64_t wide[] = {INT64_MIN, INT64_MIN + 1, -1, (int64_t)1 << 31, ((int64_t)1 << 32) + 1, (int64_t)1 << 48,
                          (int64_t)1 << 62, INT64_MAX};
  const int32_t narrow[] = {INT32_MIN, INT32_MIN + 1, -1, INT32_MAX - 1, INT32_MAX};
  for (int e = 0; e < 2; ++e) {
    const int dt = e ? HSA_STEP_BF16 : HSA_STEP_F32;
    auto quantize = [&](int64_t stride, int64_t rows, int32_t d) { return hsa_quantize_w4(dt, P(0), stride, rows, d, P(1), B(2), nullptr); };
    auto linear = [&](int32_t rows, int32_t d_in, int32_t d_out, int out) {
      return hsa_linear_w4(dt, P(0), rows, d_in, P(1), B(2), d_out, F(3), P(4), 0, out, P(5), nullptr);
    };
    auto norm = [&](int64_t qs, int64_t ks, int32_t n, int32_t heads, int32_t kv, int32_t dh, float eps, int64_t n_pos, int32_t rope,
                    int64_t qos, int64_t kos) {
      return hsa_qk_norm_rope(dt, P(0), qs, P(1), ks, n, heads, kv, dh, P(2), P(3), eps, F(4), n_pos, rope, 0, I(5), P(6), qos, P(7), kos,
                              nullptr);
    };
    for (int64_t x : wide) {
      refused(quantize(x, 10, 512), "w_stride", x);
      if (x < 0 || x > INT32_MAX) refused(quantize(512, x, 512), "n_rows", x);
      refused(norm(x, 512, 10, 8, 4, 128, 1e-6f, 100, 64, 1024, 512), "q_stride", x);
      refused(norm(1024, x, 10, 8, 4, 128, 1e-6f, 100, 64, 1024, 512), "k_stride", x);
      refused(norm(1024, 512, 10, 8, 4, 128, 1e-6f, x, 64, 1024, 512), "n_pos", x);
      refused(norm(1024, 512, 10, 8, 4, 128, 1e-6f, 100, 64, x, 512), "q_out_stride", x);
      refused(norm(1024, 512, 10, 8, 4, 128, 1e-6f, 100, 64, 1024, x), "k_out_stride", x);
    }
    for (int32_t x : narrow) {
      refused(quantize(512, 10, x), "d", x);
      refused(linear(x, 512, 100, dt), "n_rows", x);
      refused(linear(4, x, 100, dt), "d_in", x);
      refused(linear(4, 512, x, dt), "d_out", x);
      refused(linear(4, 512, 100, x), "out_dtype", x);
      refused(norm(1024, 512, x, 8, 4, 128, 1e-6f, 100, 64, 1024, 512), "n", x);
      refused(norm(1024, 512, 10, x, 4, 128, 1e-6f, 100, 64, 1024, 512), "heads", x);
      refused(norm(1024, 512, 10, 8, x, 128, 1e-6f, 100, 64, 1024, 512), "kv_heads", x);
      refused(norm(1024, 512, 10, 8, 4, x, 1e-6f, 100, 64, 1024, 512), "head_dim", x);
      refused(norm(1024, 512, 10, 8, 4, 128, 1e-6f, 100, x, 1024, 512), "rope_dim", x);
    }
    refused(quantize(512, INT32_MAX, 1 << 22), "n_rows and d", INT32_MAX);
    refused(norm(1024, 512, INT32_MAX, 1 << 15, 1 << 15, 128, 1e-6f, 100, 64, 1 << 22, 1 << 22), "n and heads", INT32_MAX);
    const float bad[] = {0.f, -1.f, INFINITY, -INFINITY, NAN, 3e38f};
    for (float x : bad) refused(norm(1024, 512, 10, 8, 4, 128, x, 100, 64, 1024, 512), "eps", 0);
    // rows in one buffer, at addresses where a difference taken as a signed number could overflow
    void* high = reinterpret_cast<void*>(UINTPTR_MAX - 0xffff);
    refused(hsa_qk_norm_rope(dt, high, 1024, P(1), 512, 10, 8, 4, 128, nullptr, nullptr, 1e-6f, F(4), 100, 64, 0, nullptr, P(1), 1024, P(7), 512,
                             nullptr), "addresses", 0);
  }
  auto plan = [&](int32_t seqs, int32_t page, int32_t pages, int32_t n_free, int32_t tokens) {
    return hsa_page_plan(I(0), I(1), seqs, page, pages, I(2), I(3), n_free, I(4), tokens, I(5), I(6), I(7), I(8), I(9), nullptr);
  };
  for (int32_t x : narrow) {
    refused(plan(x == INT32_MAX - 1 ? INT32_MIN : x, 16, 8, 100, 50), "n_seqs", x);
    refused(plan(10, x, 8, 100, 50), "page_size", x);
    refused(plan(10, 16, x, 100, 50), "max_pages", x);
    refused(plan(10, 16, 8, x, 50), "n_free", x);
    refused(plan(10, 16, 8, 100, x), "n_tokens", x);
  }
  refused(plan(INT32_MAX - 1, 1, 1 << 30, 100, 50), "n_seqs and max_pages", INT32_MAX - 1);
  if (failures) return 1;
  puts("serving_errors ok");
  return 0;
}
