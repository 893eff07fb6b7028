// Python binding of the calls over several sequences (hsa_cache_store ..
// hsa_paged_attention), whose kernels take 3 us for a small batch: what they
// check of their tensors costs 3.5 us in Python and 0.2 us here. Checks of layout, types
// and shapes, then the C entry point, whose status is returned; no computation.
//
// Every function takes the current device's index and a stream's handle first.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdio>
#include <cstdlib>
#include <exception>
#include <string>

#include "../../include/hsa_step.h"
#include "packed_tile.h"

namespace {

struct Refusal {
  PyObject* type;
  std::string what;
};
[[noreturn]] void value_error(const std::string& what) { throw Refusal{PyExc_ValueError, what}; }
[[noreturn]] void type_error(const std::string& what) { throw Refusal{PyExc_TypeError, what}; }

// The call's arguments in order.
struct Args {
  PyObject* const* at;
  Py_ssize_t n, i = 0;
  PyObject* next() {
    if (i >= n) type_error("too few arguments");
    return at[i++];
  }
  const at::Tensor* tensor_or_none() {
    PyObject* o = next();
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) type_error("expected a tensor");
    return &THPVariable_Unpack(o);
  }
  const at::Tensor& tensor() {
    const at::Tensor* t = tensor_or_none();
    if (!t) type_error("expected a tensor, got None");
    return *t;
  }
  int64_t integer() {
    const long long x = PyLong_AsLongLong(next());
    if (x == -1 && PyErr_Occurred()) throw std::exception();
    return x;
  }
  int32_t int32() {
    const int64_t x = integer();
    if (x != (int32_t)x) value_error("a size does not fit 32 bits");
    return (int32_t)x;
  }
  double real() {
    const double x = PyFloat_AsDouble(next());
    if (x == -1 && PyErr_Occurred()) throw std::exception();
    return x;
  }
  void* handle() {
    PyObject* o = next();
    void* p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw std::exception();
    return p;
  }
};

// The interpreter is free while a call enqueues, as it is in a ctypes call: a full
// queue may make it wait.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

struct Here {
  int64_t device;
  void on(const at::Tensor& t) const {
    if (!t.is_cuda()) value_error("tensors must be device tensors");
    if (t.get_device() != device)
      value_error("tensors must be on the current device (cuda:" + std::to_string(device) + "), got cuda:" +
                  std::to_string(t.get_device()));
  }
  void held(const at::Tensor& t) const {
    on(t);
    if (!t.is_contiguous()) value_error("tensors must be contiguous");
  }
  void held(const at::Tensor* t) const {
    if (t) held(*t);
  }
  void rows(const at::Tensor& t) const {
    on(t);
    if (t.dim() != 2 || t.stride(1) != 1) value_error("rows must be 2-dimensional with contiguous values");
  }
  void int32s(const at::Tensor& t) const {
    held(t);
    if (t.scalar_type() != at::kInt) type_error("indices, offsets, pages and lengths are int32");
  }
};

int dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return HSA_STEP_BF16;
  if (t.scalar_type() == at::kFloat) return HSA_STEP_F32;
  type_error("rows are bf16 or fp32");
}
void same_type(const at::Tensor& a, const at::Tensor& b) {
  if (a.scalar_type() != b.scalar_type()) type_error("rows must share one dtype");
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
const int8_t* bytes(const at::Tensor* t) { return t ? static_cast<const int8_t*>(t->data_ptr()) : nullptr; }
const int32_t* ints(const at::Tensor& t) { return static_cast<const int32_t*>(t.data_ptr()); }

// Caches of rows' dtype, or of codes with their exponents; their dtype code.
struct Caches {
  const at::Tensor &k, &v;
  const at::Tensor *k_exp, *v_exp;
  int dtype;
  int64_t n_rows, width;
};
Caches caches(const Here& here, const at::Tensor& rows, const at::Tensor& k, const at::Tensor& v, const at::Tensor* ke,
              const at::Tensor* ve, int64_t kv_heads) {
  here.held(k);
  here.held(v);
  if (k.scalar_type() != v.scalar_type() || k.dim() != 2 || k.sizes() != v.sizes())
    type_error("k_cache and v_cache must match: [n_rows, kv_heads * head_dim]");
  Caches c{k, v, nullptr, nullptr, HSA_STEP_E4M3, k.size(0), k.size(1)};
  if (k.scalar_type() != at::kFloat8_e4m3fn) {
    if (k.scalar_type() != rows.scalar_type()) type_error("caches hold the rows' dtype or float8_e4m3fn");
    c.dtype = dtype_of(rows);
  } else {
    for (const at::Tensor* e : {ke, ve}) {
      here.held(e);
      if (!e || e->scalar_type() != at::kChar || e->dim() != 2 || e->size(0) != c.n_rows || e->size(1) != kv_heads)
        type_error("float8_e4m3fn caches need int8 exponents [n_rows, kv_heads]");
    }
    c.k_exp = ke;
    c.v_exp = ve;
  }
  return c;
}

float* lse_of(const Here& here, const at::Tensor* lse, int64_t n, int64_t heads) {
  if (!lse) return nullptr;
  here.held(lse);
  if (lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != n || lse->size(1) != heads)
    type_error("lse is fp32, one value per query row and head");
  return static_cast<float*>(lse->data_ptr());
}

// (device, stream, k, v, idx, n, kv_heads, k_cache, v_cache, k_exp, v_exp)
int cache(Args& a, bool store) {
  const Here here{a.integer()};
  const hipStream_t stream = static_cast<hipStream_t>(a.handle());
  const at::Tensor &k = a.tensor(), &v = a.tensor(), &idx = a.tensor();
  const int32_t n = a.int32(), kv_heads = a.int32();
  const at::Tensor &kc = a.tensor(), &vc = a.tensor();
  const at::Tensor *ke = a.tensor_or_none(), *ve = a.tensor_or_none();
  here.rows(k);
  here.rows(v);
  here.int32s(idx);
  const int dt = dtype_of(k);
  same_type(k, v);
  const Caches c = caches(here, k, kc, vc, ke, ve, kv_heads);
  if (kv_heads < 1 || c.width % kv_heads || k.size(1) != c.width || v.size(1) != c.width || n > k.size(0) ||
      n > v.size(0) || n > idx.numel())
    value_error("k and v must hold n rows of the caches' width, a multiple of kv_heads, and idx n indices");
  const int32_t head_dim = (int32_t)(c.width / kv_heads);
  const Unlocked unlocked;
  if (store)
    return hsa_cache_store(dt, k.data_ptr(), row_stride(k), v.data_ptr(), row_stride(v), ints(idx), n, c.n_rows, kv_heads,
                           head_dim, c.dtype, kc.data_ptr(), vc.data_ptr(), const_cast<int8_t*>(bytes(c.k_exp)),
                           const_cast<int8_t*>(bytes(c.v_exp)), stream);
  return hsa_cache_load(c.dtype, kc.data_ptr(), vc.data_ptr(), bytes(c.k_exp), bytes(c.v_exp), ints(idx), n, c.n_rows,
                        kv_heads, head_dim, dt, k.data_ptr(), row_stride(k), v.data_ptr(), row_stride(v), stream);
}

// The tile that HSA_PACKED_TILE asks for, this thread's launches' until it goes.
struct Forced {
  int rows = 0, waves = 0;
  Forced() {  // with the interpreter held
    const char* tile = getenv("HSA_PACKED_TILE");
    if (!tile || !*tile) return;
    char rest;
    if (sscanf(tile, "%dx%d%c", &rows, &waves, &rest) != 2 || rows < 1 || waves < 1)
      value_error("HSA_PACKED_TILE is <rows>x<waves>, got " + std::string(tile));
    _hsa_packed_tile(rows, waves);
  }
  ~Forced() {
    if (rows) _hsa_packed_tile(0, 0);
  }
};

// (device, stream, q, k, v, cu_q, cu_kv, heads, kv_heads, head_dim, scale, causal, o, lse)
int packed(Args& a) {
  const Here here{a.integer()};
  const hipStream_t stream = static_cast<hipStream_t>(a.handle());
  const at::Tensor &q = a.tensor(), &k = a.tensor(), &v = a.tensor(), &cu_q = a.tensor(), &cu_kv = a.tensor();
  const int32_t heads = a.int32(), kv_heads = a.int32(), head_dim = a.int32();
  const float scale = (float)a.real();
  const int causal = PyObject_IsTrue(a.next());
  if (causal < 0) throw std::exception();
  const at::Tensor& o = a.tensor();
  const at::Tensor* lse = a.tensor_or_none();
  here.rows(q);
  here.rows(k);
  here.rows(v);
  here.held(o);
  here.int32s(cu_q);
  here.int32s(cu_kv);
  const int dt = dtype_of(q);
  same_type(q, k);
  same_type(q, v);
  same_type(q, o);
  float* l = lse_of(here, lse, q.size(0), heads);
  if (cu_q.numel() < 1 || cu_q.numel() > INT32_MAX || cu_kv.numel() != cu_q.numel() ||
      q.size(1) != (int64_t)heads * head_dim || o.sizes() != q.sizes() || k.size(1) != (int64_t)kv_heads * head_dim ||
      v.sizes() != k.sizes())
    value_error("q and o are [n_q, heads * head_dim], k and v [n_kv, kv_heads * head_dim], cu_q and cu_kv [n_seqs + 1]");
  const Forced forced;
  const Unlocked unlocked;
  return hsa_packed_attention(dt, q.data_ptr(), row_stride(q), k.data_ptr(), row_stride(k), v.data_ptr(), row_stride(v),
                              ints(cu_q), ints(cu_kv), (int32_t)(cu_q.numel() - 1), q.size(0), k.size(0), heads, kv_heads,
                              head_dim, scale, causal, o.data_ptr(), l, stream);
}

// (device, stream, q, k_cache, v_cache, page_table, kv_lens, page_size, heads,
//  kv_heads, head_dim, scale, o, workspace, k_exp, v_exp, lse)
int paged(Args& a) {
  const Here here{a.integer()};
  const hipStream_t stream = static_cast<hipStream_t>(a.handle());
  const at::Tensor &q = a.tensor(), &kc = a.tensor(), &vc = a.tensor(), &table = a.tensor(), &lens = a.tensor();
  const int32_t page_size = a.int32(), heads = a.int32(), kv_heads = a.int32(), head_dim = a.int32();
  const float scale = (float)a.real();
  const at::Tensor& o = a.tensor();
  const at::Tensor *ws = a.tensor_or_none(), *ke = a.tensor_or_none(), *ve = a.tensor_or_none();
  const at::Tensor* lse = a.tensor_or_none();
  here.rows(q);
  here.held(o);
  here.held(ws);
  here.int32s(table);
  here.int32s(lens);
  const int dt = dtype_of(q);
  same_type(q, o);
  const Caches c = caches(here, q, kc, vc, ke, ve, kv_heads);
  float* l = lse_of(here, lse, q.size(0), heads);
  if (page_size < 1 || table.dim() != 2 || table.size(0) != q.size(0) || table.size(1) > INT32_MAX ||
      lens.numel() != q.size(0) || q.size(0) > INT32_MAX || q.size(1) != (int64_t)heads * head_dim ||
      o.sizes() != q.sizes() || c.width != (int64_t)kv_heads * head_dim || c.n_rows / page_size > INT32_MAX)
    value_error("q and o are [n_seqs, heads * head_dim], the caches [n_rows, kv_heads * head_dim], page_table "
                "[n_seqs, max_pages], kv_lens [n_seqs], page_size at least 1");
  const Unlocked unlocked;
  return hsa_paged_attention(dt, q.data_ptr(), row_stride(q), c.dtype, kc.data_ptr(), vc.data_ptr(), bytes(c.k_exp),
                             bytes(c.v_exp), ints(table), (int32_t)table.size(1), ints(lens), (int32_t)q.size(0),
                             (int32_t)(c.n_rows / page_size), page_size, heads, kv_heads, head_dim, scale, o.data_ptr(), l,
                             ws ? ws->data_ptr() : nullptr, ws ? ws->numel() * ws->element_size() : 0, stream);
}

template <class F>
PyObject* call(PyObject* const* at, Py_ssize_t n, F f) {
  try {
    Args a{at, n};
    const int status = f(a);
    return PyLong_FromLong(status);
  } catch (const Refusal& r) {
    PyErr_SetString(r.type, r.what.c_str());
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

PyObject* cache_store(PyObject*, PyObject* const* at, Py_ssize_t n) {
  return call(at, n, [](Args& a) { return cache(a, true); });
}
PyObject* cache_load(PyObject*, PyObject* const* at, Py_ssize_t n) {
  return call(at, n, [](Args& a) { return cache(a, false); });
}
PyObject* packed_attention(PyObject*, PyObject* const* at, Py_ssize_t n) { return call(at, n, packed); }
PyObject* paged_attention(PyObject*, PyObject* const* at, Py_ssize_t n) { return call(at, n, paged); }

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {{"cache_store", fast(cache_store), METH_FASTCALL, nullptr},
                         {"cache_load", fast(cache_load), METH_FASTCALL, nullptr},
                         {"packed_attention", fast(packed_attention), METH_FASTCALL, nullptr},
                         {"paged_attention", fast(paged_attention), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seq_binding() { return PyModule_Create(&module); }
