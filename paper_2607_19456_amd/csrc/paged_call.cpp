// paged_call.cpp -- the arguments of the paged calls, of prompt attention and of the
// rotation by several axes, taken apart in C++.
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
decltype(&da_prompt_attn) g_prompt;
decltype(&da_prompt_attn_grad) g_prompt_grad;
decltype(&da_rotary_axes) g_rotary;

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

int type_of(const Tensor& t) {
  const at::ScalarType type = t.scalar_type();
  return type == at::kFloat ? DA_F32 : type == at::kBFloat16 ? DA_BF16
         : type == at::kHalf ? DA_F16 : -1;
}

// The starts of packed sequences, or NULL; *B: how many sequences, 0 if not known.
bool starts(PyObject* o, long most, long gpu, const int32_t** p, int64_t* B) {
  *p = nullptr;
  if (o == Py_None) return true;
  const Tensor* t = whole(o, at::kInt, gpu);
  if (!t || t->dim() != 1 || t->size(0) < 2 || most < 1 || (*B && *B != t->size(0) - 1)) return false;
  *p = static_cast<const int32_t*>(t->data_ptr());
  *B = t->size(0) - 1;
  return true;
}

// The packed sequences that q, k, the starts and T and N describe.
bool prompt(PyObject* q_, PyObject* k_, PyObject* row_start, long T, PyObject* key_start, long N,
            int causal, long gpu, da_prompt* p) {
  if (!THPVariable_Check(q_) || !THPVariable_Check(k_)) return false;
  const Tensor &q = THPVariable_Unpack(q_), &k = THPVariable_Unpack(k_);
  if (q.dim() != 3 || k.dim() != 3 || type_of(q) < 0 || T < 0 || N < 0) return false;
  const int64_t rows = q.size(0), keys = k.size(0);
  if (key_start == Py_None && N == 0 && row_start != Py_None && keys == rows)
    key_start = row_start, N = T;
  const int32_t *rs, *ks;
  int64_t B = 0;
  if (!starts(row_start, T, gpu, &rs, &B) || !starts(key_start, N, gpu, &ks, &B)) return false;
  if (!rs) {
    if (!B) B = T > 0 ? rows / T : 1;
    if (B < 1) return false;
    if (!T) T = rows / B;
    if (rows != B * T) return false;
  }
  if (!ks) {
    if (!N) N = keys / B;
    if (keys != B * N) return false;
  }
  for (int64_t x : {B, q.size(1), k.size(1), q.size(2), rows, keys, (int64_t)T, (int64_t)N})
    if (!fits(x)) return false;
  *p = {rs, ks, (int)B, (int)q.size(1), (int)k.size(1), (int)q.size(2),
        (int)rows, (int)keys, (int)T, (int)N, type_of(q), causal};
  return true;
}

// [rows][h_q] float, contiguous.
const Tensor* statistics(PyObject* o, const da_prompt& p, long gpu) {
  const Tensor* t = whole(o, at::kFloat, gpu);
  return t && t->dim() == 2 && t->size(0) == p.rows && t->size(1) == p.h_q ? t : nullptr;
}

// prompt(q, k, v, scale, causal, row_start, T, key_start, N, out, lse, workspace, gpu, stream)
PyObject* prompt_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return not_here();
  const double scale = PyFloat_AsDouble(a[3]);
  const long T = PyLong_AsLong(a[6]), N = PyLong_AsLong(a[8]), gpu = PyLong_AsLong(a[12]);
  void* stream = PyLong_AsVoidPtr(a[13]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return not_here();
  }
  const int causal = truth(a[4]);
  da_prompt p;
  if (causal < 0 || !prompt(a[0], a[1], a[5], T, a[7], N, causal, gpu, &p)) return not_here();
  const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
  int64_t qs, ks, vs;
  const Tensor* q = tokens(a[0], type, gpu, p.rows, p.h_q, p.d, &qs);
  const Tensor* k = tokens(a[1], type, gpu, p.keys, p.h_kv, p.d, &ks);
  const Tensor* v = tokens(a[2], type, gpu, p.keys, p.h_kv, p.d, &vs);
  const Tensor* out = whole(a[9], type, gpu);
  const Tensor* lse = a[10] == Py_None ? nullptr : statistics(a[10], p, gpu);
  const Tensor* ws = whole(a[11], at::kByte, gpu);
  if (!q || !k || !v || !out || out->sizes() != q->sizes() || (a[10] != Py_None && !lse) || !ws)
    return not_here();
  return PyLong_FromLong(g_prompt(&p, q->data_ptr(), qs, k->data_ptr(), ks, v->data_ptr(), vs,
                                  (float)scale, out->data_ptr(),
                                  lse ? static_cast<float*>(lse->data_ptr()) : nullptr,
                                  ws->data_ptr(), (size_t)ws->numel(), stream));
}

// prompt_grad(q, k, v, out, lse, d_out, scale, causal, row_start, T, key_start, N, dq, dk, dv,
//             workspace, gpu, stream)
PyObject* prompt_grad_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 18) return not_here();
  const double scale = PyFloat_AsDouble(a[6]);
  const long T = PyLong_AsLong(a[9]), N = PyLong_AsLong(a[11]), gpu = PyLong_AsLong(a[16]);
  void* stream = PyLong_AsVoidPtr(a[17]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return not_here();
  }
  const int causal = truth(a[7]);
  da_prompt p;
  if (causal < 0 || !prompt(a[0], a[1], a[8], T, a[10], N, causal, gpu, &p)) return not_here();
  const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
  int64_t qs, ks, vs, gs, dqs, dks, dvs;
  const Tensor* q = tokens(a[0], type, gpu, p.rows, p.h_q, p.d, &qs);
  const Tensor* k = tokens(a[1], type, gpu, p.keys, p.h_kv, p.d, &ks);
  const Tensor* v = tokens(a[2], type, gpu, p.keys, p.h_kv, p.d, &vs);
  const Tensor* out = whole(a[3], type, gpu);
  const Tensor* lse = statistics(a[4], p, gpu);
  const Tensor* g = tokens(a[5], type, gpu, p.rows, p.h_q, p.d, &gs);
  const Tensor* dq = tokens(a[12], type, gpu, p.rows, p.h_q, p.d, &dqs);
  const Tensor* dk = tokens(a[13], type, gpu, p.keys, p.h_kv, p.d, &dks);
  const Tensor* dv = tokens(a[14], type, gpu, p.keys, p.h_kv, p.d, &dvs);
  const Tensor* ws = whole(a[15], at::kByte, gpu);
  if (!q || !k || !v || !out || out->sizes() != q->sizes() || !lse || !g || !dq || !dk || !dv ||
      !ws)
    return not_here();
  return PyLong_FromLong(g_prompt_grad(
      &p, q->data_ptr(), qs, k->data_ptr(), ks, v->data_ptr(), vs, out->data_ptr(),
      static_cast<const float*>(lse->data_ptr()), g->data_ptr(), gs, (float)scale, dq->data_ptr(),
      dqs, dk->data_ptr(), dks, dv->data_ptr(), dvs, ws->data_ptr(), (size_t)ws->numel(), stream));
}

// rotary(q, positions, table, sections, k, interleaved, inverse, q_out, k_out, gpu, stream)
PyObject* rotary_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !THPVariable_Check(a[0])) return not_here();
  const long gpu = PyLong_AsLong(a[9]);
  void* stream = PyLong_AsVoidPtr(a[10]);
  const bool is_list = PyList_Check(a[3]);
  if (PyErr_Occurred() || (!is_list && !PyTuple_Check(a[3]))) {
    PyErr_Clear();
    return not_here();
  }
  const Py_ssize_t axes = is_list ? PyList_GET_SIZE(a[3]) : PyTuple_GET_SIZE(a[3]);
  const int interleaved = truth(a[5]), inverse = truth(a[6]);
  const Tensor& like = THPVariable_Unpack(a[0]);
  const Tensor *pos = whole(a[1], at::kInt, gpu), *table = whole(a[2], at::kFloat, gpu);
  if (axes < 1 || axes > 4 || interleaved < 0 || inverse < 0 || like.dim() != 3 ||
      type_of(like) < 0 || !pos || pos->dim() != 2 || !table || table->dim() != 2)
    return not_here();
  const at::ScalarType type = like.scalar_type();
  const int64_t rows = like.size(0), h_q = like.size(1), d = like.size(2);
  int64_t h_kv = 0, qs, qos, ks = 0, kos = 0;
  const Tensor* q = tokens(a[0], type, gpu, rows, h_q, d, &qs);
  const Tensor* q_out = tokens(a[7], type, gpu, rows, h_q, d, &qos);
  const Tensor *k = nullptr, *k_out = nullptr;
  if (a[4] != Py_None) {
    if (!THPVariable_Check(a[4]) || THPVariable_Unpack(a[4]).dim() != 3) return not_here();
    h_kv = THPVariable_Unpack(a[4]).size(1);
    k = tokens(a[4], type, gpu, rows, h_kv, d, &ks);
    k_out = tokens(a[8], type, gpu, rows, h_kv, d, &kos);
    if (!k || !k_out) return not_here();
  }
  if (!q || !q_out || pos->size(0) != axes || pos->size(1) != rows) return not_here();
  for (int64_t x : {rows, h_q, h_kv, d, table->size(0), table->size(1)})
    if (!fits(x)) return not_here();
  da_rotary p = {static_cast<const int32_t*>(pos->data_ptr()),
                 static_cast<const float*>(table->data_ptr()), (int)rows, (int)d, type_of(like),
                 (int)table->size(0), (int)table->size(1), (int)axes, {0, 0, 0, 0}, interleaved,
                 inverse};
  for (Py_ssize_t x = 0; x < axes; ++x) {
    PyObject* o = is_list ? PyList_GET_ITEM(a[3], x) : PyTuple_GET_ITEM(a[3], x);
    const long section = PyLong_Check(o) ? PyLong_AsLong(o) : -1;
    if (!fits(section)) {
      PyErr_Clear();
      return not_here();
    }
    p.sections[x] = (int)section;
  }
  return PyLong_FromLong(g_rotary(&p, q->data_ptr(), qs, (int)h_q, q_out->data_ptr(), qos,
                                  k ? k->data_ptr() : nullptr, ks, (int)h_kv,
                                  k ? k_out->data_ptr() : nullptr, kos, stream));
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

// use(append, gather, attn, prompt, prompt_grad, rotary): the addresses of the C ABI's
// functions.
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "use(append, gather, attn, prompt, prompt_grad, rotary)");
    return nullptr;
  }
  g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[0]));
  g_gather = reinterpret_cast<decltype(g_gather)>(PyLong_AsVoidPtr(a[1]));
  g_attn = reinterpret_cast<decltype(g_attn)>(PyLong_AsVoidPtr(a[2]));
  g_prompt = reinterpret_cast<decltype(g_prompt)>(PyLong_AsVoidPtr(a[3]));
  g_prompt_grad = reinterpret_cast<decltype(g_prompt_grad)>(PyLong_AsVoidPtr(a[4]));
  g_rotary = reinterpret_cast<decltype(g_rotary)>(PyLong_AsVoidPtr(a[5]));
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
    {"prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<prompt_call>)),
     METH_FASTCALL, ""},
    {"prompt_grad",
     reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<prompt_grad_call>)),
     METH_FASTCALL, ""},
    {"rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<rotary_call>)),
     METH_FASTCALL, ""},
    {"use", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(use)), METH_FASTCALL, ""},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "paged_call", nullptr, -1, kMethods,
                       nullptr,               nullptr,      nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_paged_call() { return PyModule_Create(&kModule); }
