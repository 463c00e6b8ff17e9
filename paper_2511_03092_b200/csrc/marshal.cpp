// Argument marshalling of the rotary and paged-cache calls: checks that the tensors of a call are what the library is
// told they are and passes their addresses on.  A serving step makes these calls once per layer, and the same checks
// cost 5 to 10 us a call as Python expressions, more than the kernels of a small step take.
//
// Every function takes the address of the library's entry point, the structures (ctypes objects, read through the buffer
// protocol), the tensors or None, and the stream's handle or None for the current one.  It returns the entry point's
// status, or None when a tensor is not what it should be (nothing was called; the caller finds the words).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "snapstream.h"

namespace {

using at::Tensor;
using Sizes = std::initializer_list<int64_t>;

// A structure handed over as a ctypes object.
template <typename S> struct Struct {
  Py_buffer view{};
  const S* p = nullptr;
  bool ok = true;
  explicit Struct(PyObject* o) {
    if (o == Py_None) return;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) { ok = false; return; }
    if (view.len == (Py_ssize_t)sizeof(S)) p = static_cast<const S*>(view.buf);
    else { ok = false; PyErr_SetString(PyExc_TypeError, "not the structure that this call takes"); }
  }
  ~Struct() { if (view.obj) PyBuffer_Release(&view); }
};

struct Call {
  PyObject* const* args;
  bool good = true;               // every tensor so far is what it should be
  int device = -2;                // -2: no tensor yet
  const Tensor* at(int i) {
    if (args[i] == Py_None) return nullptr;
    if (!THPVariable_Check(args[i])) { good = false; return nullptr; }
    return &THPVariable_Unpack(args[i]);
  }
  const Tensor* any(int i) {
    const Tensor* t = at(i);
    if (!t) return nullptr;
    const int d = t->is_cuda() ? t->get_device() : -1;
    if (device == -2) device = d;
    good = good && d == device && d >= 0;
    return t;
  }
  // a dense tensor of this type and shape, or None
  void* dense(int i, at::ScalarType type, at::IntArrayRef shape) {
    const Tensor* t = any(i);
    if (!t) return nullptr;
    good = good && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous();
    return good ? t->data_ptr() : nullptr;
  }
  // ... of this type and any shape
  void* dense(int i, at::ScalarType type) {
    const Tensor* t = any(i);
    if (!t) return nullptr;
    good = good && t->scalar_type() == type && t->is_contiguous();
    return good ? t->data_ptr() : nullptr;
  }
  // a [tokens][heads][d] tensor of any strides, the last dim dense
  void* rows(int i, at::ScalarType type, at::IntArrayRef shape, int64_t (&stride)[2]) {
    stride[0] = stride[1] = 0;
    const Tensor* t = any(i);
    if (!t) return nullptr;
    good = good && t->scalar_type() == type && t->sizes() == shape && t->stride(2) == 1;
    if (!good) return nullptr;
    stride[0] = t->stride(0); stride[1] = t->stride(1);
    return t->data_ptr();
  }
  void* pages(int i, at::ScalarType type, at::IntArrayRef shape, at::IntArrayRef strides) {
    const Tensor* t = any(i);
    if (!t) { good = false; return nullptr; }
    good = good && t->scalar_type() == type && t->sizes() == shape && t->strides() == strides;
    return good ? t->data_ptr() : nullptr;
  }
  void need(const void* p) { good = good && p; }
  // The stream to launch on; the tensors have to be on the current device.
  void* stream(PyObject* o) {
    if (device < 0 || device != (int)c10::cuda::current_device()) { good = false; return nullptr; }
    if (o != Py_None) return PyLong_AsVoidPtr(o);
    return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  }
};

at::ScalarType type_of(const snap_config_t* c) { return c->dtype == SNAP_F32 ? at::kFloat : at::kBFloat16; }

PyObject* answer(const Call& c, int status) {
  if (PyErr_Occurred()) return nullptr;
  if (!c.good) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

// The parts of a paged call that all three share: pages, table, lengths, status.
struct PagedParts { void* k; void* v; int32_t* table; int32_t* seq_len; uint32_t* status; };
PagedParts paged_parts(Call& c, const snap_config_t* cfg, const snap_paged_t* p, int k, int v, int table, int seq_len, int status) {
  PagedParts r;
  const at::ScalarType t = type_of(cfg);
  r.k = c.pages(k, t, Sizes{p->n_pages, cfg->n_kv_heads, p->page_tokens, cfg->d_qk}, Sizes{p->k_page_stride, p->k_head_stride, p->k_row_stride, 1});
  r.v = c.pages(v, t, Sizes{p->n_pages, cfg->n_kv_heads, p->page_tokens, cfg->d_v}, Sizes{p->v_page_stride, p->v_head_stride, p->v_row_stride, 1});
  c.need(r.table = static_cast<int32_t*>(c.dense(table, at::kInt, Sizes{cfg->max_seqs, p->max_pages})));
  c.need(r.seq_len = static_cast<int32_t*>(c.dense(seq_len, at::kInt, Sizes{cfg->max_seqs})));
  r.status = static_cast<uint32_t*>(c.dense(status, at::kInt));
  return r;
}
float* weights(Call& c, int i, const snap_config_t* cfg, const snap_paged_t* p) {
  return static_cast<float*>(c.dense(i, at::kFloat, Sizes{cfg->max_seqs, cfg->n_kv_heads, (int64_t)p->max_pages * p->page_tokens}));
}
int32_t* ints(Call& c, int i, int64_t n) { return static_cast<int32_t*>(c.dense(i, at::kInt, Sizes{n})); }
// scratch: any dense tensor
void* scratch(Call& c, int i, size_t& bytes) {
  const Tensor* t = c.any(i);
  c.good = c.good && t && t->is_contiguous();
  bytes = c.good ? t->nbytes() : 0;
  return c.good ? t->data_ptr() : nullptr;
}
// Counts are passed on as 32-bit integers.
int64_t countable(Call& c, int64_t n) {
  c.good = c.good && n <= INT32_MAX;
  return n;
}
int64_t length(Call& c, int i) {
  const Tensor* t = c.at(i);
  if (t && t->dim() == 1) return countable(c, t->size(0));
  c.good = false;
  return 0;
}

// entry, cfg, rope, freqs, positions, q, k, q_out, k_out, inverse, stream
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!count(n_args, 11)) return nullptr;
  const auto fn = reinterpret_cast<decltype(&snap_rope)>(PyLong_AsVoidPtr(a[0]));
  Struct<snap_config_t> cfg(a[1]);
  Struct<snap_rope_config_t> rp(a[2]);
  if (!fn || !cfg.ok || !rp.ok) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_TypeError, "no entry point"), nullptr);
  if (!cfg.p || !rp.p) return PyLong_FromLong(SNAP_ERR_NULL_POINTER);
  Call c{a};
  const int64_t n = length(c, 4), hq = cfg.p->n_q_heads, hkv = cfg.p->n_kv_heads, d = cfg.p->d_qk;
  const at::ScalarType t = type_of(cfg.p);
  int64_t qs[2], ks[2], qos[2], kos[2];
  const double* freqs = static_cast<const double*>(c.dense(3, at::kDouble, Sizes{rp.p->rot_dim / 2}));
  const int32_t* pos = ints(c, 4, n);
  void* q = c.rows(5, t, Sizes{n, hq, d}, qs);
  void* k = c.rows(6, t, Sizes{n, hkv, d}, ks);
  void* qo = c.rows(7, t, Sizes{n, hq, d}, qos);
  void* ko = c.rows(8, t, Sizes{n, hkv, d}, kos);
  const int inverse = (int)PyLong_AsLong(a[9]);
  void* st = c.stream(a[10]);
  int rc = 0;
  if (c.good && !PyErr_Occurred())
    rc = fn(cfg.p, rp.p, freqs, pos, (int32_t)n, q, qs[0], qs[1], qo, qos[0], qos[1], k, ks[0], ks[1], ko, kos[0], kos[1], inverse, st);
  return answer(c, rc);
}

// entry, cfg, paged, slots, rows, k, v, k_pages, v_pages, table, seq_len, rope, freqs, positions, q, q_out, k_out, weights, status, stream
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!count(n_args, 20)) return nullptr;
  const auto fn = reinterpret_cast<decltype(&snap_paged_append)>(PyLong_AsVoidPtr(a[0]));
  Struct<snap_config_t> cfg(a[1]);
  Struct<snap_paged_t> p(a[2]);
  Struct<snap_rope_config_t> rp(a[11]);
  if (!fn || !cfg.ok || !p.ok || !rp.ok) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_TypeError, "no entry point"), nullptr);
  if (!cfg.p || !p.p) return PyLong_FromLong(SNAP_ERR_NULL_POINTER);
  Call c{a};
  const int64_t n = length(c, 3), hq = cfg.p->n_q_heads, hkv = cfg.p->n_kv_heads, d = cfg.p->d_qk;
  const at::ScalarType t = type_of(cfg.p);
  const PagedParts pp = paged_parts(c, cfg.p, p.p, 7, 8, 9, 10, 18);
  int64_t ks[2], vs[2], qs[2];
  const int32_t* slots = ints(c, 3, n);
  const int32_t* rows = ints(c, 4, n);
  void* k = c.rows(5, t, Sizes{n, hkv, d}, ks);
  void* v = c.rows(6, t, Sizes{n, hkv, cfg.p->d_v}, vs);
  const double* freqs = rp.p ? static_cast<const double*>(c.dense(12, at::kDouble, Sizes{rp.p->rot_dim / 2})) : nullptr;
  const int32_t* pos = rp.p ? ints(c, 13, n) : nullptr;
  void* q = c.rows(14, t, Sizes{n, hq, d}, qs);
  void* qo = c.dense(15, t, Sizes{n, hq, d});
  void* ko = c.dense(16, t, Sizes{n, hkv, d});
  float* w = weights(c, 17, cfg.p, p.p);
  void* st = c.stream(a[19]);
  int rc = 0;
  if (c.good && !PyErr_Occurred())
    rc = fn(cfg.p, p.p, slots, rows, (int32_t)n, rp.p, freqs, pos, q, qs[0], qs[1], qo, k, ks[0], ks[1], ko, v, vs[0], vs[1], pp.k, pp.v, pp.table,
            pp.seq_len, w, pp.status, st);
  return answer(c, rc);
}

// entry, cfg, paged, q, slots, n, k_pages, v_pages, table, seq_len, out, workspace, weights_in, weights_out, status, stream
PyObject* paged_decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!count(n_args, 16)) return nullptr;
  const auto fn = reinterpret_cast<decltype(&snap_paged_decode_attn)>(PyLong_AsVoidPtr(a[0]));
  Struct<snap_config_t> cfg(a[1]);
  Struct<snap_paged_t> p(a[2]);
  if (!fn || !cfg.ok || !p.ok) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_TypeError, "no entry point"), nullptr);
  if (!cfg.p || !p.p) return PyLong_FromLong(SNAP_ERR_NULL_POINTER);
  Call c{a};
  const int64_t n = countable(c, PyLong_AsLong(a[5])), hq = cfg.p->n_q_heads;
  const at::ScalarType t = type_of(cfg.p);
  const PagedParts pp = paged_parts(c, cfg.p, p.p, 6, 7, 8, 9, 14);
  size_t bytes;
  void* q = c.dense(3, t, Sizes{n, hq, cfg.p->d_qk});
  const int32_t* slots = ints(c, 4, n);
  void* out = c.dense(10, t, Sizes{n, hq, cfg.p->d_v});
  void* ws = scratch(c, 11, bytes);
  float* wi = weights(c, 12, cfg.p, p.p);
  float* wo = weights(c, 13, cfg.p, p.p);
  void* st = c.stream(a[15]);
  int rc = 0;
  if (c.good && !PyErr_Occurred())
    rc = fn(cfg.p, p.p, q, slots, (int32_t)n, pp.k, pp.v, pp.table, pp.seq_len, wi, wo, out, ws, bytes, pp.status, st);
  return answer(c, rc);
}

// entry, cfg, paged, src, dst, n, k_pages, v_pages, table, seq_len, weights_in, weights_out, workspace, kept_rows, status, stream
PyObject* paged_evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (!count(n_args, 16)) return nullptr;
  const auto fn = reinterpret_cast<decltype(&snap_paged_evict)>(PyLong_AsVoidPtr(a[0]));
  Struct<snap_config_t> cfg(a[1]);
  Struct<snap_paged_t> p(a[2]);
  if (!fn || !cfg.ok || !p.ok) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_TypeError, "no entry point"), nullptr);
  if (!cfg.p || !p.p) return PyLong_FromLong(SNAP_ERR_NULL_POINTER);
  Call c{a};
  const int64_t n = countable(c, PyLong_AsLong(a[5]));
  const PagedParts pp = paged_parts(c, cfg.p, p.p, 6, 7, 8, 9, 14);
  size_t bytes;
  const int32_t* src = ints(c, 3, n);
  const int32_t* dst = ints(c, 4, n);
  float* wi = weights(c, 10, cfg.p, p.p);
  float* wo = weights(c, 11, cfg.p, p.p);
  void* ws = scratch(c, 12, bytes);
  int32_t* kept = static_cast<int32_t*>(c.dense(13, at::kInt, Sizes{n, cfg.p->n_kv_heads, (int64_t)cfg.p->l_sink + cfg.p->topk + cfg.p->l_recent}));
  void* st = c.stream(a[15]);
  int rc = 0;
  if (c.good && !PyErr_Occurred())
    rc = fn(cfg.p, p.p, src, dst, (int32_t)n, pp.k, pp.v, pp.table, pp.seq_len, wi, wo, kept, ws, bytes, pp.status, st);
  return answer(c, rc);
}

// What torch or the language runtime throws becomes a Python error.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(self, args, n);
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
    return nullptr;
  }
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction method() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F>)); }

PyMethodDef methods[] = {{"rope", method<rope>(), METH_FASTCALL, nullptr},
                         {"paged_append", method<paged_append>(), METH_FASTCALL, nullptr},
                         {"paged_decode_attn", method<paged_decode_attn>(), METH_FASTCALL, nullptr},
                         {"paged_evict", method<paged_evict>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the rotary and paged-cache calls.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef BUILT_FOR_TORCH
#define BUILT_FOR_TORCH "unknown"
#endif
// Tensors are read through torch's own classes, so the module fits one torch only; the build looks for this line in the file.
const char built_for[] = "built for torch " BUILT_FOR_TORCH;

PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", built_for + sizeof("built for torch ") - 1) != 0) { Py_DECREF(m); return nullptr; }
  return m;
}
