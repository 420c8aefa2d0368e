// paged_call.cpp -- the paged calls' arguments, taken apart in C++.
//
// A decode step makes two calls a layer, whose kernels take 3 to 10 us on small
// batches; looking at ten tensors from Python takes as long (0.1 us an
// attribute).  These functions look at the same things and call the C ABI.  They
// know only calls that are right: for anything else they return -1 before any
// work, and the caller goes its own way, which names the error.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "decode_attn.h"

namespace {

decltype(&da_paged_append) g_append;
decltype(&da_paged_gather) g_gather;
decltype(&da_paged_attn) g_attn;

using at::Tensor;

const Tensor* tensor(PyObject* o, at::ScalarType type, long gpu) {
  if (!THPVariable_Check(o)) return nullptr;
  const Tensor& t = THPVariable_Unpack(o);
  return t.layout() == at::kStrided && t.scalar_type() == type && t.is_cuda() &&
                 t.get_device() == gpu
             ? &t
             : nullptr;
}

const Tensor* whole(PyObject* o, at::ScalarType type, long gpu) {
  const Tensor* t = tensor(o, type, gpu);
  return t && t->is_contiguous() ? t : nullptr;
}

// [rows][heads][d], a token's heads contiguous; *stride between tokens.
const Tensor* tokens(PyObject* o, at::ScalarType type, long gpu, int64_t rows, int64_t heads,
                     int64_t d, int64_t* stride) {
  const Tensor* t = tensor(o, type, gpu);
  if (!t || t->dim() != 3 || t->size(0) != rows || t->size(1) != heads || t->size(2) != d)
    return nullptr;
  if ((t->stride(2) != 1) || (t->stride(1) != d && heads != 1)) return nullptr;
  *stride = rows > 1 ? t->stride(0) : heads * d;
  return t;
}

bool fits(int64_t x) { return x >= 0 && x <= INT32_MAX; }

// The batch that K, V, pages, past, row_start and T describe with rows of
// `like`'s type and size d.
bool batch(PyObject* const* a, PyObject* row_start, long T, long gpu, const Tensor& like,
           da_paged_kv* kv) {
  if (!THPVariable_Check(a[0])) return false;
  const at::ScalarType type = like.scalar_type();
  const int dtype = type == at::kFloat ? DA_F32 : type == at::kBFloat16 ? DA_BF16
                    : type == at::kHalf ? DA_F16 : -1;
  const bool mx4 = THPVariable_Unpack(a[0]).scalar_type() == at::kByte;
  const at::ScalarType pool = mx4 ? at::kByte : type;
  const Tensor *K = whole(a[0], pool, gpu), *V = whole(a[1], pool, gpu);
  const Tensor *pages = whole(a[2], at::kInt, gpu), *past = whole(a[3], at::kInt, gpu);
  if (dtype < 0 || !K || !V || !pages || !past || K->dim() != 4 || K->sizes() != V->sizes() ||
      pages->dim() != 2 || past->dim() != 1 || past->size(0) != pages->size(0))
    return false;
  const int64_t d = like.size(2), rows = like.size(0), B = pages->size(0);
  if (K->size(3) != (mx4 ? d / 2 + d / 32 : d)) return false;
  const void* start = nullptr;
  if (row_start != Py_None) {
    const Tensor* s = whole(row_start, at::kInt, gpu);
    if (!s || s->dim() != 1 || s->size(0) != B + 1 || T < 1) return false;
    start = s->data_ptr();
  } else {
    if (T == 0 && B) T = rows / B;
    if (rows != B * T) return false;
  }
  for (int64_t x : {B, K->size(0), K->size(1), K->size(2), d, pages->size(1), rows, (int64_t)T})
    if (!fits(x)) return false;
  *kv = {K->data_ptr(), V->data_ptr(), static_cast<const int32_t*>(pages->data_ptr()),
         static_cast<const int32_t*>(past->data_ptr()), static_cast<const int32_t*>(start),
         (int)B, (int)K->size(1), (int)d, (int)K->size(0), (int)K->size(2), (int)pages->size(1),
         (int)rows, (int)T, dtype, mx4 ? DA_KV_MX4 : DA_KV_DENSE};
  return true;
}

PyObject* not_here() { return PyLong_FromLong(-1); }

// 1 or 0, or -1 for what has no truth value.
int truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) PyErr_Clear();
  return t;
}

// append(K, V, pages, past, k_new, v_new, q, rotary, interleaved, row_start, T, q_out, gpu,
//        stream)
PyObject* append_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 14 || !THPVariable_Check(a[4])) return not_here();
  const long T = PyLong_AsLong(a[10]), gpu = PyLong_AsLong(a[12]);
  void* stream = PyLong_AsVoidPtr(a[13]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return not_here();
  }
  const int interleaved = truth(a[8]);
  if (interleaved < 0) return not_here();
  const Tensor& like = THPVariable_Unpack(a[4]);
  da_paged_kv kv;
  if (like.dim() != 3 || !batch(a, a[9], T, gpu, like, &kv)) return not_here();
  const at::ScalarType type = like.scalar_type();
  int64_t ks, vs, qs = 0;
  const Tensor* k = tokens(a[4], type, gpu, kv.rows, kv.h_kv, kv.d, &ks);
  const Tensor* v = tokens(a[5], type, gpu, kv.rows, kv.h_kv, kv.d, &vs);
  if (!k || !v) return not_here();
  const Tensor *q = nullptr, *out = nullptr, *rotary = nullptr;
  if (a[6] != Py_None) {
    if (!THPVariable_Check(a[6]) || THPVariable_Unpack(a[6]).dim() != 3) return not_here();
    q = tokens(a[6], type, gpu, kv.rows, THPVariable_Unpack(a[6]).size(1), kv.d, &qs);
    out = whole(a[11], type, gpu);
    if (!q || !out || out->sizes() != q->sizes() || !fits(q->size(1))) return not_here();
  }
  if (a[7] != Py_None) {
    rotary = whole(a[7], at::kFloat, gpu);
    if (!rotary || rotary->dim() != 2 || !fits(rotary->size(0)) || !fits(rotary->size(1)))
      return not_here();
  }
  return PyLong_FromLong(g_append(
      &kv, k->data_ptr(), v->data_ptr(), ks, vs, q ? q->data_ptr() : nullptr, qs,
      q ? (int)q->size(1) : 0, q ? out->data_ptr() : nullptr,
      rotary ? static_cast<const float*>(rotary->data_ptr()) : nullptr,
      rotary ? (int)rotary->size(0) : 0, rotary ? (int)rotary->size(1) : 0,
      interleaved, stream));
}

// gather(K, V, pages, past, k_out, v_out, row_start, T, gpu, stream)
PyObject* gather_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 10 || !THPVariable_Check(a[4])) return not_here();
  const long T = PyLong_AsLong(a[7]), gpu = PyLong_AsLong(a[8]);
  void* stream = PyLong_AsVoidPtr(a[9]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return not_here();
  }
  const Tensor& like = THPVariable_Unpack(a[4]);
  da_paged_kv kv;
  if (like.dim() != 3 || !batch(a, a[6], T, gpu, like, &kv)) return not_here();
  const Tensor *k = whole(a[4], like.scalar_type(), gpu), *v = whole(a[5], like.scalar_type(), gpu);
  if (!k || !v || k->size(1) != kv.h_kv || v->sizes() != k->sizes()) return not_here();
  return PyLong_FromLong(g_gather(&kv, k->data_ptr(), v->data_ptr(), stream));
}

// attn(K, V, pages, past, q, scale, causal, row_start, T, out, workspace, gpu, stream)
PyObject* attn_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 13 || !THPVariable_Check(a[4])) return not_here();
  const long T = PyLong_AsLong(a[8]), gpu = PyLong_AsLong(a[11]);
  const double scale = PyFloat_AsDouble(a[5]);
  void* stream = PyLong_AsVoidPtr(a[12]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return not_here();
  }
  const int causal = truth(a[6]);
  if (causal < 0) return not_here();
  const Tensor& like = THPVariable_Unpack(a[4]);
  da_paged_kv kv;
  if (like.dim() != 3 || !batch(a, a[7], T, gpu, like, &kv) || !fits(like.size(1)))
    return not_here();
  int64_t qs;
  const Tensor* q = tokens(a[4], like.scalar_type(), gpu, kv.rows, like.size(1), kv.d, &qs);
  const Tensor* out = whole(a[9], like.scalar_type(), gpu);
  const Tensor* ws = whole(a[10], at::kByte, gpu);
  if (!q || !out || !ws || out->sizes() != q->sizes()) return not_here();
  return PyLong_FromLong(g_attn(&kv, q->data_ptr(), qs, (int)q->size(1), (float)scale,
                                causal, out->data_ptr(), ws->data_ptr(),
                                (size_t)ws->numel(), stream));
}

// (What torch throws, say for a tensor without storage, is not for here either.)
template <PyObject* (*call)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return call(a, n);
  } catch (...) {
    return not_here();
  }
}

// use(append, gather, attn): the addresses of the C ABI's functions.
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "use(append, gather, attn)");
    return nullptr;
  }
  g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[0]));
  g_gather = reinterpret_cast<decltype(g_gather)>(PyLong_AsVoidPtr(a[1]));
  g_attn = reinterpret_cast<decltype(g_attn)>(PyLong_AsVoidPtr(a[2]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<append_call>)),
     METH_FASTCALL, ""},
    {"gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<gather_call>)),
     METH_FASTCALL, ""},
    {"attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<attn_call>)),
     METH_FASTCALL, ""},
    {"use", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(use)), METH_FASTCALL, ""},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "paged_call", nullptr, -1, kMethods,
                       nullptr,               nullptr,      nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_paged_call() { return PyModule_Create(&kModule); }
