// C ABI entry points of the calls over several sequences: host-side argument
// checks, then kernel launches. See include/hsa_step.h for their contract.
#include "api_util.h"
#include "seq_common.h"

using namespace hsa_api;

namespace {

constexpr int64_t kMaxStride = int64_t(1) << 22;  // elements between rows
constexpr int64_t kMaxKeys = int64_t(1) << 30;    // keys of a sequence, so that a position plus a block fits an int
constexpr int64_t kMaxLaunch = int64_t(1) << 32;  // threads of one launch
constexpr int64_t kMaxW4Rows = int64_t(1) << 18;  // fewer than 2^16 tiles of 5 rows, a launch's second dimension

// Bytes from the first to the end of the last of n rows `stride` elements apart.
size_t span(int64_t n, int64_t stride, int64_t width, size_t es) {
  return n > 0 ? ((size_t)(n - 1) * (size_t)stride + (size_t)width) * es : 0;
}

// Rows of a strided input: their stride and alignment (bf16 16 bytes, fp32 4).
bool rows_ok(const void* p, int64_t n, int64_t stride, int64_t width, size_t es) {
  if (stride < width || stride > kMaxStride || !fits(n, stride, es)) return false;
  return es == 2 ? aligned(p, 16) && stride % 8 == 0 : aligned(p, 4);
}

bool heads_ok(int32_t heads, int32_t kv_heads, int32_t head_dim) {
  return heads > 0 && kv_heads > 0 && heads % kv_heads == 0 && (head_dim == 64 || head_dim == 128) &&
         (int64_t)heads * head_dim <= kMaxStride;
}

// the kernels take scale * log2(e) in fp32
bool scale_ok(float scale) { return scale > 0.f && scale <= 0x1p127f; }

struct Range {
  const void* p;
  size_t n;
};

// True if the first `outs` ranges overlap each other or any later range.
template <int N>
bool any_overlap(const Range (&r)[N], int outs) {
  for (int i = 0; i < outs; ++i)
    for (int j = i + 1; j < N; ++j)
      if (overlaps(r[i].p, r[i].n, r[j].p, r[j].n)) return true;
  return false;
}

// How a cache holds rows of kv_heads heads: the bytes of a row (0 unless cache_dtype is
// dtype or a type of codes), its exponents, and the alignment of its first row.
struct HeldRow {
  hsa::Held held;
  size_t bytes, exps, align;
};
HeldRow held_row(int dtype, int cache_dtype, int64_t kv_heads, int64_t head_dim) {
  const size_t d = (size_t)(kv_heads * head_dim);
  if (cache_dtype == HSA_STEP_E4M3) return {hsa::kE4M3, d, (size_t)kv_heads, 16};
  if (cache_dtype == HSA_STEP_E2M1) return {hsa::kE2M1, d / 2, d / hsa::kGroup, 16};
  const size_t es = cache_dtype == dtype ? elem_size(dtype) : 0;
  return {hsa::kOwn, d * es, 0, es == 4 ? size_t(4) : size_t(16)};
}
bool cache_dtype_ok(int dtype, int cache_dtype) {
  return elem_size(dtype) && (cache_dtype == dtype || cache_dtype == HSA_STEP_E4M3 || cache_dtype == HSA_STEP_E2M1);
}

// Checks of hsa_cache_store and hsa_cache_load that do not depend on the direction.
int check_cache(int dtype, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                const int32_t* idx, int32_t n, int64_t n_rows, int32_t kv_heads, int32_t head_dim,
                int cache_dtype, const void* k_cache, const void* v_cache, const int8_t* k_exp,
                const int8_t* v_exp) {
  if (!cache_dtype_ok(dtype, cache_dtype)) return HSA_STEP_ERR_DTYPE;
  const size_t es = elem_size(dtype);
  if (n < 0 || n_rows < 0 || n_rows > kMaxRows || !heads_ok(kv_heads, kv_heads, head_dim)) return HSA_STEP_ERR_SHAPE;
  const int64_t d = (int64_t)kv_heads * head_dim;
  const HeldRow row = held_row(dtype, cache_dtype, kv_heads, head_dim);
  // one launch: fewer than 2^32 threads of 8 values
  if (!fits(n_rows, (int64_t)row.bytes) || (int64_t)n * d >= kMaxLaunch * 4) return HSA_STEP_ERR_SHAPE;
  if (n == 0) return HSA_STEP_OK;
  if (!k || !v || !idx || (n_rows > 0 && (!k_cache || !v_cache))) return HSA_STEP_ERR_NULL;
  if (row.exps && n_rows > 0 && (!k_exp || !v_exp)) return HSA_STEP_ERR_NULL;
  if (!rows_ok(k, n, k_stride, d, es) || !rows_ok(v, n, v_stride, d, es) || !aligned(idx, 4) ||
      !aligned(k_cache, row.align) || !aligned(v_cache, row.align))
    return HSA_STEP_ERR_SHAPE;
  return HSA_STEP_OK;
}

}  // namespace

HSA_API int hsa_cache_store(int dtype, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride, const int32_t* idx, int32_t n, int64_t n_rows,
                            int32_t kv_heads, int32_t head_dim, int cache_dtype, void* k_cache,
                            void* v_cache, int8_t* k_exp, int8_t* v_exp, hipStream_t stream) {
  const int st = check_cache(dtype, k, k_stride, v, v_stride, idx, n, n_rows, kv_heads, head_dim,
                             cache_dtype, k_cache, v_cache, k_exp, v_exp);
  if (st != HSA_STEP_OK || n == 0) return st;
  const int64_t d = (int64_t)kv_heads * head_dim;
  const HeldRow row = held_row(dtype, cache_dtype, kv_heads, head_dim);
  const size_t cb = (size_t)n_rows * row.bytes, eb = (size_t)n_rows * row.exps;
  const size_t es = elem_size(dtype);
  const Range r[] = {{k_cache, cb}, {v_cache, cb}, {k_exp, eb}, {v_exp, eb}, {k, span(n, k_stride, d, es)},
                     {v, span(n, v_stride, d, es)}, {idx, (size_t)n * 4}};
  if (any_overlap(r, 4)) return HSA_STEP_ERR_ALIAS;
  if (n_rows == 0) return HSA_STEP_OK;
  hsa::CacheRows c{};
  c.bf16 = dtype == HSA_STEP_BF16;
  c.held = row.held;
  c.src_k = k;
  c.src_v = v;
  c.dst_k = k_cache;
  c.dst_v = v_cache;
  c.k_exp = k_exp;
  c.v_exp = v_exp;
  c.k_stride = k_stride;
  c.v_stride = v_stride;
  c.idx = idx;
  c.n = n;
  c.n_rows = n_rows;
  c.kv_heads = kv_heads;
  c.head_dim = head_dim;
  return launch_status(hsa::launch_cache_store(c, stream));
}

HSA_API int hsa_cache_load(int cache_dtype, const void* k_cache, const void* v_cache,
                           const int8_t* k_exp, const int8_t* v_exp, const int32_t* idx, int32_t n,
                           int64_t n_rows, int32_t kv_heads, int32_t head_dim, int dtype, void* k,
                           int64_t k_stride, void* v, int64_t v_stride, hipStream_t stream) {
  const int st = check_cache(dtype, k, k_stride, v, v_stride, idx, n, n_rows, kv_heads, head_dim,
                             cache_dtype, k_cache, v_cache, k_exp, v_exp);
  if (st != HSA_STEP_OK || n == 0) return st;
  const int64_t d = (int64_t)kv_heads * head_dim;
  const HeldRow row = held_row(dtype, cache_dtype, kv_heads, head_dim);
  const size_t cb = (size_t)n_rows * row.bytes, eb = (size_t)n_rows * row.exps;
  const size_t es = elem_size(dtype);
  const Range r[] = {{k, span(n, k_stride, d, es)}, {v, span(n, v_stride, d, es)}, {k_cache, cb}, {v_cache, cb},
                     {k_exp, eb}, {v_exp, eb}, {idx, (size_t)n * 4}};
  if (any_overlap(r, 2)) return HSA_STEP_ERR_ALIAS;
  hsa::CacheRows c{};
  c.bf16 = dtype == HSA_STEP_BF16;
  c.held = row.held;
  c.src_k = k_cache;
  c.src_v = v_cache;
  c.dst_k = k;
  c.dst_v = v;
  c.k_exp = const_cast<int8_t*>(k_exp);
  c.v_exp = const_cast<int8_t*>(v_exp);
  c.k_stride = k_stride;
  c.v_stride = v_stride;
  c.idx = idx;
  c.n = n;
  c.n_rows = n_rows;
  c.kv_heads = kv_heads;
  c.head_dim = head_dim;
  return launch_status(hsa::launch_cache_load(c, stream));
}

HSA_API int hsa_packed_attention(int dtype, const void* q, int64_t q_stride, const void* k,
                                 int64_t k_stride, const void* v, int64_t v_stride,
                                 const int32_t* cu_q, const int32_t* cu_kv, int32_t n_seqs,
                                 int64_t n_q, int64_t n_kv, int32_t heads, int32_t kv_heads,
                                 int32_t head_dim, float scale, int32_t causal, void* o, float* lse,
                                 hipStream_t stream) {
  const size_t es = elem_size(dtype);
  if (!es) return HSA_STEP_ERR_DTYPE;
  if (!heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || n_seqs == INT32_MAX || n_q < 0 || n_kv < 0 ||
      n_q > kMaxRows / heads || n_kv > kMaxKeys || !scale_ok(scale))
    return HSA_STEP_ERR_SHAPE;
  // one launch: fewer than 2^32 threads, 512 per 16 rows or item
  if (n_q * heads / 16 + ((int64_t)n_seqs + 8) * kv_heads >= kMaxLaunch / 512) return HSA_STEP_ERR_SHAPE;
  if (n_q == 0 || n_seqs == 0) return HSA_STEP_OK;
  if (!q || !cu_q || !cu_kv || !o || (n_kv > 0 && (!k || !v))) return HSA_STEP_ERR_NULL;
  const int64_t d = (int64_t)heads * head_dim, dk = (int64_t)kv_heads * head_dim;
  if (!rows_ok(q, n_q, q_stride, d, es) || (n_kv > 0 && (!rows_ok(k, n_kv, k_stride, dk, es) || !rows_ok(v, n_kv, v_stride, dk, es))) ||
      !aligned(o, es == 2 ? 16 : 4) || !aligned(lse, 4) || !aligned(cu_q, 4) || !aligned(cu_kv, 4))
    return HSA_STEP_ERR_SHAPE;
  const size_t cub = ((size_t)n_seqs + 1) * 4;
  const Range r[] = {{o, (size_t)n_q * d * es}, {lse, lse ? (size_t)n_q * heads * 4 : 0}, {q, span(n_q, q_stride, d, es)},
                     {k, span(n_kv, k_stride, dk, es)}, {v, span(n_kv, v_stride, dk, es)}, {cu_q, cub}, {cu_kv, cub}};
  if (any_overlap(r, 2)) return HSA_STEP_ERR_ALIAS;
  hsa::PackedArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.cu_q = cu_q;
  a.cu_kv = cu_kv;
  a.n_seqs = n_seqs;
  a.n_q = (int)n_q;
  a.n_kv = (int)n_kv;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.by_group = hsa::FastDiv((uint32_t)a.group);
  a.scale = scale;
  a.causal = causal != 0;
  a.o = o;
  a.lse = lse;
  return launch_status(hsa::launch_packed_attention(a, dtype == HSA_STEP_BF16, head_dim, stream));
}

HSA_API size_t hsa_paged_attention_workspace_bytes(int dtype, int32_t n_seqs, int32_t heads,
                                                   int32_t kv_heads, int32_t head_dim,
                                                   int64_t max_len) {
  if (!elem_size(dtype) || !heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || max_len < 0 ||
      max_len > kMaxKeys || n_seqs > kMaxRows / heads)
    return 0;
  // for any cache: e2m1 rows take the most
  return hsa::paged_attention_bytes(n_seqs, kv_heads, heads / kv_heads, head_dim, max_len, true);
}

HSA_API int hsa_paged_attention(int dtype, const void* q, int64_t q_stride, int cache_dtype,
                                const void* k_cache, const void* v_cache, const int8_t* k_exp,
                                const int8_t* v_exp, const int32_t* page_table, int32_t max_pages,
                                const int32_t* kv_lens, int32_t n_seqs, int32_t n_pages,
                                int32_t page_size, int32_t heads, int32_t kv_heads,
                                int32_t head_dim, float scale, void* o, float* lse,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!cache_dtype_ok(dtype, cache_dtype)) return HSA_STEP_ERR_DTYPE;
  const size_t es = elem_size(dtype);
  if (!heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || n_seqs > kMaxRows / heads || n_pages < 0 ||
      max_pages < 0 || page_size < 1 || (int64_t)n_pages * page_size > kMaxRows ||
      (int64_t)max_pages * page_size > kMaxKeys || !scale_ok(scale))
    return HSA_STEP_ERR_SHAPE;
  const int64_t d = (int64_t)heads * head_dim;
  const HeldRow row = held_row(dtype, cache_dtype, kv_heads, head_dim);
  const int64_t n_rows = (int64_t)n_pages * page_size;
  if (!fits(n_rows, (int64_t)row.bytes) || !fits(n_seqs, max_pages, 4) || (int64_t)n_seqs * heads >= kMaxLaunch / 512)
    return HSA_STEP_ERR_SHAPE;
  if (n_seqs == 0) return HSA_STEP_OK;
  if (!q || !kv_lens || !o || (max_pages > 0 && !page_table) || (n_rows > 0 && (!k_cache || !v_cache)) ||
      (row.exps && n_rows > 0 && (!k_exp || !v_exp)))
    return HSA_STEP_ERR_NULL;
  if (!rows_ok(q, n_seqs, q_stride, d, es) || !aligned(k_cache, row.align) || !aligned(v_cache, row.align) ||
      !aligned(o, es == 2 ? 16 : 4) || !aligned(lse, 4) || !aligned(page_table, 4) || !aligned(kv_lens, 4))
    return HSA_STEP_ERR_SHAPE;
  const size_t need = hsa::paged_attention_bytes(n_seqs, kv_heads, heads / kv_heads, head_dim, (long)max_pages * page_size,
                                                 row.held == hsa::kE2M1);
  if (need && (!workspace || workspace_bytes < need)) return HSA_STEP_ERR_WORKSPACE;
  if (need && !aligned(workspace, 16)) return HSA_STEP_ERR_SHAPE;
  const size_t cb = (size_t)n_rows * row.bytes, eb = (size_t)n_rows * row.exps;
  const Range r[] = {{o, (size_t)n_seqs * d * es}, {lse, lse ? (size_t)n_seqs * heads * 4 : 0}, {workspace, need},
                     {q, span(n_seqs, q_stride, d, es)}, {k_cache, cb}, {v_cache, cb}, {k_exp, eb}, {v_exp, eb},
                     {page_table, (size_t)n_seqs * max_pages * 4}, {kv_lens, (size_t)n_seqs * 4}};
  if (any_overlap(r, 3)) return HSA_STEP_ERR_ALIAS;
  hsa::PagedArgs a{};
  a.q = q;
  a.q_stride = q_stride;
  a.k = k_cache;
  a.v = v_cache;
  a.k_exp = k_exp;
  a.v_exp = v_exp;
  a.page_table = page_table;
  a.kv_lens = kv_lens;
  a.max_pages = max_pages;
  a.n_seqs = n_seqs;
  a.n_pages = n_pages;
  a.page_size = page_size;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.scale = scale;
  a.o = o;
  a.lse = lse;
  a.ws = workspace;
  return launch_status(hsa::launch_paged_attention(a, dtype == HSA_STEP_BF16, row.held, head_dim, stream));
}

HSA_API int hsa_quantize_w4(int dtype, const void* w, int64_t w_stride, int64_t n_rows, int32_t d, void* codes,
                            int8_t* exps, hipStream_t stream) {
  const size_t es = elem_size(dtype);
  if (!es) return HSA_STEP_ERR_DTYPE;
  // one launch: fewer than 2^32 threads of 8 values
  if (n_rows < 0 || n_rows > kMaxRows || d < 1 || d > kMaxStride || d % hsa::kGroup != 0 || n_rows * d >= kMaxLaunch * 8 - 2048)
    return HSA_STEP_ERR_SHAPE;
  if (n_rows == 0) return HSA_STEP_OK;
  if (!w || !codes || !exps) return HSA_STEP_ERR_NULL;
  if (!rows_ok(w, n_rows, w_stride, d, es) || !aligned(codes, 16)) return HSA_STEP_ERR_SHAPE;
  const Range r[] = {{codes, (size_t)n_rows * d / 2}, {exps, (size_t)n_rows * d / hsa::kGroup}, {w, span(n_rows, w_stride, d, es)}};
  if (any_overlap(r, 2)) return HSA_STEP_ERR_ALIAS;
  return launch_status(hsa::launch_quantize_w4(w, dtype == HSA_STEP_BF16, n_rows, d, w_stride, codes, exps, stream));
}

HSA_API int hsa_linear_w4(int dtype, const void* x, int32_t n_rows, int32_t d_in, const void* w, const int8_t* w_exp,
                          int32_t d_out, const float* row_scale, const void* residual, int32_t gelu, int out_dtype,
                          void* y, hipStream_t stream) {
  const size_t es = elem_size(dtype), os = elem_size(out_dtype);
  if (!es || (out_dtype != dtype && !(dtype == HSA_STEP_BF16 && out_dtype == HSA_STEP_F32))) return HSA_STEP_ERR_DTYPE;
  if (n_rows < 0 || d_in < 1 || d_in > kMaxStride || d_in % hsa::kGroup != 0 || d_out < 0 || d_out > kMaxStride ||
      n_rows > kMaxW4Rows)
    return HSA_STEP_ERR_SHAPE;
  if ((gelu && residual) || (out_dtype != dtype && (gelu || residual))) return HSA_STEP_ERR_SHAPE;
  if (n_rows == 0 || d_out == 0) return HSA_STEP_OK;
  if (!x || !w || !w_exp || !y) return HSA_STEP_ERR_NULL;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(y, 16) || !aligned(residual, 16) || !aligned(row_scale, 4))
    return HSA_STEP_ERR_SHAPE;
  const size_t yb = (size_t)n_rows * d_out * os;
  const Range r[] = {{y, yb}, {x, (size_t)n_rows * d_in * es}, {w, (size_t)d_out * d_in / 2},
                     {w_exp, (size_t)d_out * d_in / hsa::kGroup}, {row_scale, row_scale ? (size_t)n_rows * 4 : 0},
                     {residual, residual && residual != y ? yb : 0}};
  if (any_overlap(r, 1)) return HSA_STEP_ERR_ALIAS;
  hsa::LinearW4 a{};
  a.x = x;
  a.w = static_cast<const uint8_t*>(w);
  a.exps = w_exp;
  a.rows = n_rows;
  a.d_in = d_in;
  a.d_out = d_out;
  a.row_scale = row_scale;
  a.residual = residual;
  a.gelu = gelu != 0;
  a.out_f32 = out_dtype != dtype;
  a.y = y;
  return launch_status(hsa::launch_linear_w4(a, dtype == HSA_STEP_BF16, stream));
}

HSA_API int hsa_qk_norm_rope(int dtype, const void* q, int64_t q_stride, const void* k, int64_t k_stride, int32_t n,
                             int32_t heads, int32_t kv_heads, int32_t head_dim, const void* q_weight,
                             const void* k_weight, float eps, const float* rope, int64_t n_pos, int32_t rope_dim,
                             int32_t interleaved, const int32_t* pos, void* q_out, int64_t q_out_stride, void* k_out,
                             int64_t k_out_stride, hipStream_t stream) {
  const size_t es = elem_size(dtype);
  if (!es) return HSA_STEP_ERR_DTYPE;
  if (n < 0 || heads < 0 || kv_heads < 0 || (head_dim != 64 && head_dim != 128) ||
      (int64_t)heads * head_dim > kMaxStride || (int64_t)kv_heads * head_dim > kMaxStride || !(eps > 0.f) || eps > 0x1p127f ||
      rope_dim < 0 || rope_dim > head_dim || rope_dim % 8 != 0 || n_pos < 0 || n_pos > kMaxRows)
    return HSA_STEP_ERR_SHAPE;
  const int64_t d = (int64_t)heads * head_dim, dk = (int64_t)kv_heads * head_dim;
  // one launch: fewer than 2^32 threads of 8 values
  if ((__int128)n * (d + dk) >= kMaxLaunch * 8 - 2048) return HSA_STEP_ERR_SHAPE;
  if (n == 0 || heads + (int64_t)kv_heads == 0) return HSA_STEP_OK;
  if ((heads > 0 && (!q || !q_out)) || (kv_heads > 0 && (!k || !k_out)) || (rope_dim > 0 && n_pos > 0 && !rope))
    return HSA_STEP_ERR_NULL;
  if ((heads > 0 && (!rows_ok(q, n, q_stride, d, es) || !rows_ok(q_out, n, q_out_stride, d, es))) ||
      (kv_heads > 0 && (!rows_ok(k, n, k_stride, dk, es) || !rows_ok(k_out, n, k_out_stride, dk, es))))
    return HSA_STEP_ERR_SHAPE;
  const size_t wa = es == 2 ? 16 : 4;
  if (!aligned(q_weight, wa) || !aligned(k_weight, wa) || !aligned(rope, 16) || !aligned(pos, 4)) return HSA_STEP_ERR_SHAPE;
  const size_t qb = heads > 0 ? span(n, q_stride, d, es) : 0, kb = kv_heads > 0 ? span(n, k_stride, dk, es) : 0;
  const size_t qob = heads > 0 ? span(n, q_out_stride, d, es) : 0, kob = kv_heads > 0 ? span(n, k_out_stride, dk, es) : 0;
  // queries and keys lie in one projection's output, between each other's rows: their rows may not
  // meet, their spans may
  auto meet = [&](const void* p, int64_t ps, int64_t pw, size_t pb, const void* o, int64_t os, int64_t ow, size_t ob) {
    if (!overlaps(p, pb, o, ob)) return false;
    if (ps != os) return true;
    const int64_t row = ps * (int64_t)es;
    int64_t at = (int64_t)(reinterpret_cast<uintptr_t>(o) - reinterpret_cast<uintptr_t>(p)) % row;
    if (at < 0) at += row;
    return n > 1 ? at < pw * (int64_t)es || at + ow * (int64_t)es > row : true;
  };
  const bool q_here = q == q_out && q_stride == q_out_stride, k_here = k == k_out && k_stride == k_out_stride;
  if (heads > 0 && ((!q_here && meet(q, q_stride, d, qb, q_out, q_out_stride, d, qob)) ||
                    (kv_heads > 0 && meet(k, k_stride, dk, kb, q_out, q_out_stride, d, qob))))
    return HSA_STEP_ERR_ALIAS;
  if (kv_heads > 0 && ((!k_here && meet(k, k_stride, dk, kb, k_out, k_out_stride, dk, kob)) ||
                       (heads > 0 && meet(q, q_stride, d, qb, k_out, k_out_stride, dk, kob))))
    return HSA_STEP_ERR_ALIAS;
  if (heads > 0 && kv_heads > 0 && meet(q_out, q_out_stride, d, qob, k_out, k_out_stride, dk, kob)) return HSA_STEP_ERR_ALIAS;
  const size_t wb = (size_t)head_dim * es, rb = rope_dim ? (size_t)n_pos * rope_dim * 4 : 0, pb = pos ? (size_t)n * 4 : 0;
  const Range r[] = {{heads > 0 ? q_out : nullptr, qob}, {kv_heads > 0 ? k_out : nullptr, kob}, {q_weight, wb}, {k_weight, wb},
                     {rope, rb}, {pos, pb}};
  for (int o = 0; o < 2; ++o)
    for (int i = 2; i < 6; ++i)
      if (overlaps(r[o].p, r[o].n, r[i].p, r[i].n)) return HSA_STEP_ERR_ALIAS;
  hsa::NormRope a{};
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.qo_stride = q_out_stride;
  a.ko_stride = k_out_stride;
  a.n = n;
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.eps = eps;
  a.rope = rope;
  a.rope_dim = n_pos > 0 ? rope_dim : 0;
  a.interleaved = interleaved != 0;
  a.n_pos = n_pos;
  a.pos = pos;
  return launch_status(hsa::launch_norm_rope(a, dtype == HSA_STEP_BF16, head_dim, stream));
}

HSA_API int hsa_page_plan(const int32_t* past, const int32_t* fresh, int32_t n_seqs, int32_t page_size, int32_t max_pages,
                          int32_t* page_table, const int32_t* free_pages, int32_t n_free, const int32_t* free_at,
                          int32_t n_tokens, int32_t* cu, int32_t* kv_lens, int32_t* pos, int32_t* slots,
                          int32_t* free_next, hipStream_t stream) {
  if (n_seqs < 0 || n_seqs == INT32_MAX || page_size < 1 || max_pages < 0 || (int64_t)max_pages * page_size > kMaxKeys || n_free < 0 ||
      n_free > kMaxKeys || n_tokens < 0 || n_tokens >= kMaxKeys || !fits(n_seqs, max_pages, 4))
    return HSA_STEP_ERR_SHAPE;
  if ((n_seqs > 0 && (!past || !fresh || !kv_lens || (max_pages > 0 && !page_table))) || (n_free > 0 && !free_pages) ||
      !free_at || !free_next || !cu || (n_tokens > 0 && (!pos || !slots)))
    return HSA_STEP_ERR_NULL;
  const void* ints[] = {past, fresh, page_table, free_pages, free_at, cu, kv_lens, pos, slots, free_next};
  for (const void* p : ints)
    if (!aligned(p, 4)) return HSA_STEP_ERR_SHAPE;
  const size_t sb = (size_t)n_seqs * 4, tb = (size_t)n_tokens * 4;
  // kv_lens may be past, free_next free_at: a step that goes on from the last one's
  const Range r[] = {{page_table, (size_t)n_seqs * max_pages * 4}, {cu, sb + 4}, {kv_lens, sb}, {pos, tb}, {slots, tb}, {free_next, 12},
                     {kv_lens == past ? nullptr : past, sb}, {fresh, sb}, {free_pages, (size_t)n_free * 4},
                     {free_at == free_next ? nullptr : free_at, 12}};
  if (any_overlap(r, 6)) return HSA_STEP_ERR_ALIAS;
  hsa::PagePlan a{};
  a.past = past;
  a.fresh = fresh;
  a.n_seqs = n_seqs;
  a.page_size = page_size;
  a.max_pages = max_pages;
  a.page_table = page_table;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.free_at = free_at;
  a.n_tokens = n_tokens;
  a.cu = cu;
  a.kv_lens = kv_lens;
  a.pos = pos;
  a.slots = slots;
  a.free_next = free_next;
  return launch_status(hsa::launch_page_plan(a, stream));
}
