// Host-side argument checks of the calls over several sequences under
// AddressSanitizer and UndefinedBehaviorSanitizer (built by
// tests/test_seq_sanitize.py with the library's host code instrumented). Every
// call is refused on the host before anything is enqueued, or has nothing to
// do; pointers are fake device addresses that are never dereferenced. Each size
// argument takes the extremes of its type in turn, where a product of sizes in a
// check could overflow.
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

int main() {
  const int64_t wide[] = {INT64_MIN, INT64_MIN + 1, -1, (int64_t)1 << 31, ((int64_t)1 << 32) + 1, (int64_t)1 << 48,
                          (int64_t)1 << 62, INT64_MAX};
  const int32_t narrow[] = {INT32_MIN, INT32_MIN + 1, -1, INT32_MAX - 1, INT32_MAX};
  for (int e = 0; e < 2; ++e) {
    const int dt = e ? HSA_STEP_BF16 : HSA_STEP_F32;
    auto store = [&](int64_t ks, int64_t vs, int32_t n, int64_t rows, int32_t kv, int32_t dh, int cd) {
      const int a = hsa_cache_store(dt, P(0), ks, P(1), vs, (int32_t*)P(2), n, rows, kv, dh, cd, P(3), P(4),
                                    (int8_t*)P(5), (int8_t*)P(6), nullptr);
      const int b = hsa_cache_load(cd, P(3), P(4), (int8_t*)P(5), (int8_t*)P(6), (int32_t*)P(2), n, rows, kv, dh, dt,
                                   P(0), ks, P(1), vs, nullptr);
      return a == b ? a : HSA_STEP_ERR_LAUNCH;
    };
    for (int64_t x : wide) {
      refused(store(x, 512, 10, 100, 4, 128, HSA_STEP_E4M3), "k_stride", x);
      refused(store(512, x, 10, 100, 4, 128, HSA_STEP_E4M3), "v_stride", x);
      refused(store(512, 512, 10, x, 4, 128, dt), "n_rows", x);
    }
    for (int32_t x : narrow) {
      refused(store(512, 512, x, 100, 4, 128, HSA_STEP_E4M3), "n", x);
      refused(store(512, 512, 10, 100, x, 128, HSA_STEP_E4M3), "kv_heads", x);
      refused(store(512, 512, 10, 100, 4, x, HSA_STEP_E4M3), "head_dim", x);
      refused(store(512, 512, 10, 100, 4, 128, x), "cache_dtype", x);
    }
    auto packed = [&](int64_t qs, int64_t ks, int32_t seqs, int64_t nq, int64_t nk, int32_t heads, int32_t kv, int32_t dh,
                      float scale) {
      return hsa_packed_attention(dt, P(0), qs, P(1), ks, P(2), ks, (int32_t*)P(3), (int32_t*)P(4), seqs, nq, nk, heads, kv,
                                  dh, scale, 1, P(5), (float*)P(6), nullptr);
    };
    for (int64_t x : wide) {
      refused(packed(x, 512, 3, 100, 100, 8, 4, 128, 0.1f), "q_stride", x);
      refused(packed(1024, x, 3, 100, 100, 8, 4, 128, 0.1f), "k_stride", x);
      refused(packed(1024, 512, 3, x, 100, 8, 4, 128, 0.1f), "n_q", x);
      refused(packed(1024, 512, 3, 100, x, 8, 4, 128, 0.1f), "n_kv", x);
    }
    for (int32_t x : narrow) {
      refused(packed(1024, 512, x, 100, 100, 8, 4, 128, 0.1f), "n_seqs", x);
      refused(packed(1024, 512, 3, 100, 100, x, 4, 128, 0.1f), "heads", x);
      refused(packed(1024, 512, 3, 100, 100, 8, x, 128, 0.1f), "kv_heads", x);
      refused(packed(1024, 512, 3, 100, 100, x, x, 128, 0.1f), "heads = kv_heads", x);
      refused(packed(1024, 512, 3, 100, 100, 8, 4, x, 0.1f), "head_dim", x);
    }
    auto paged = [&](int64_t qs, int32_t most, int32_t seqs, int32_t pages, int32_t page, int32_t heads, int32_t kv,
                     int32_t dh, size_t ws) {
      return hsa_paged_attention(dt, P(0), qs, HSA_STEP_E4M3, P(1), P(2), (int8_t*)P(3), (int8_t*)P(4), (int32_t*)P(5),
                                 most, (int32_t*)P(6), seqs, pages, page, heads, kv, dh, 0.1f, P(7), (float*)P(8), P(9), ws,
                                 nullptr);
    };
    for (int64_t x : wide) refused(paged(x, 100, 3, 100, 64, 8, 4, 128, 32 << 20), "q_stride", x);
    for (int32_t x : narrow) {
      refused(paged(1024, x, 3, 100, 64, 8, 4, 128, 32 << 20), "max_pages", x);
      refused(paged(1024, 100, x, 100, 64, 8, 4, 128, 32 << 20), "n_seqs", x);
      refused(paged(1024, 100, 3, x, 64, 8, 4, 128, 32 << 20), "n_pages", x);
      refused(paged(1024, 100, 3, 100, x, 8, 4, 128, 32 << 20), "page_size", x);
      refused(paged(1024, 100, 3, 100, 64, x, 4, 128, 32 << 20), "heads", x);
      refused(paged(1024, 100, 3, 100, 64, 8, x, 128, 32 << 20), "kv_heads", x);
      refused(paged(1024, 100, 3, 100, 64, 8, 4, x, 32 << 20), "head_dim", x);
    }
    refused(paged(1024, 100, 3, 100, 64, 8, 4, 128, 0), "workspace_bytes", 0);
    for (int64_t x : wide)
      if (hsa_paged_attention_workspace_bytes(dt, 3, 8, 4, 128, x) != 0) ++failures;
    for (int32_t x : narrow) {
      if (hsa_paged_attention_workspace_bytes(dt, x, 8, 4, 128, 10000) != 0) ++failures;
      if (hsa_paged_attention_workspace_bytes(dt, 3, x, x, 128, 10000) != 0) ++failures;
      if (hsa_paged_attention_workspace_bytes(dt, 3, 8, 4, x, 10000) != 0) ++failures;
    }
    if (hsa_paged_attention_workspace_bytes(dt, 1 << 20, 4, 4, 128, 1 << 30) > HSA_STEP_PAGED_WORKSPACE_BYTES) ++failures;
  }
  if (failures) return 1;
  printf("seq_errors ok\n");
  return 0;
}
