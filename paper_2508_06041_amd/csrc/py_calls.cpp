// The calls a program makes per linear, layer and token, for Python: dpllm_gemv and dpllm_estimate, and those around the linears.  What binding.py does
// through ctypes, without a Python object per argument.  us of host time per call of a loop, ctypes -> here: dpllm_gemv 4.3 -> 3.4, of which the
// launch is 2.5.
// A call that is out of the ordinary in any way (an argument that is no int or has no data_ptr(), a closed model) is not made here:
// the answer is kElsewhere and binding.py makes it the long way, with the errors that has.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <initializer_list>

#include "../../include/dpllm.h"

namespace {

constexpr long kElsewhere = 1;

using Gemv = int (*)(void*, int, int, const int32_t*, const void*, void*, int, void*);
using Estimate = int (*)(void*, int, int, int, const void*, float*, int32_t*, void*);
Gemv the_gemv = nullptr;
Estimate the_estimate = nullptr;
PyObject *get_device = nullptr, *get_stream = nullptr;   // torch._C._cuda_getDevice, _cuda_getCurrentRawStream
PyObject *s_data_ptr = nullptr, *s_dim = nullptr, *s_size = nullptr, *zero = nullptr;

// A C int as ctypes converts one; false: no int.
bool as_int(PyObject* o, int* v) {
  if (!PyLong_Check(o)) return false;
  *v = (int)PyLong_AsUnsignedLongMask(o);
  return true;
}

// false: not to be had (no error is left behind)
bool address(PyObject* o, void** p) {
  PyObject* a = PyLong_Check(o) ? Py_NewRef(o) : PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (a != nullptr && PyLong_Check(a)) {
    *p = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    if (!PyErr_Occurred()) return true;
  } else {
    Py_XDECREF(a);
  }
  PyErr_Clear();
  return false;
}

bool tensor(PyObject* o, void** p) { return !PyLong_Check(o) && address(o, p); }

// the current stream of the current device, and that device
bool stream(void** p, int* device = nullptr) {
  PyObject* d = PyObject_CallNoArgs(get_device);
  PyObject* s = d != nullptr ? PyObject_CallOneArg(get_stream, d) : nullptr;
  const bool ok = s != nullptr && PyLong_Check(s) && (device == nullptr || as_int(d, device));
  if (ok) *p = PyLong_AsVoidPtr(s);
  Py_XDECREF(d);
  Py_XDECREF(s);
  if (!ok || PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}

// samples of x: 1 for a vector, else its first dimension
bool samples(PyObject* x, int* n) {
  PyObject* d = PyObject_CallMethodNoArgs(x, s_dim);
  int dim = 0;
  bool ok = d != nullptr && as_int(d, &dim);
  Py_XDECREF(d);
  *n = 1;
  if (ok && dim != 1) {
    PyObject* s = PyObject_CallMethodOneArg(x, s_size, zero);
    ok = s != nullptr && as_int(s, n);
    Py_XDECREF(s);
  }
  if (!ok) PyErr_Clear();
  return ok;
}

// bind(address of dpllm_gemv, of dpllm_estimate, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *g = nullptr, *e = nullptr;
  if (n != 4 || !address(a[0], &g) || !address(a[1], &e)) {
    PyErr_SetString(PyExc_TypeError, "bind(gemv, estimate, get_device, get_stream)");
    return nullptr;
  }
  the_gemv = reinterpret_cast<Gemv>(g);
  the_estimate = reinterpret_cast<Estimate>(e);
  Py_XSETREF(get_device, Py_NewRef(a[2]));
  Py_XSETREF(get_stream, Py_NewRef(a[3]));
  Py_RETURN_NONE;
}

// gemv(model, id, k, x, y, k_dev or None)
PyObject* gemv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *m = nullptr, *x = nullptr, *y = nullptr, *kd = nullptr, *st = nullptr;
  int id = 0, k = 0, b = 0;
  if (n != 6 || the_gemv == nullptr || !PyLong_Check(a[0]) || !address(a[0], &m) || m == nullptr || !as_int(a[1], &id) || !as_int(a[2], &k) ||
      !tensor(a[3], &x) || !tensor(a[4], &y) || (a[5] != Py_None && !tensor(a[5], &kd)) || !samples(a[3], &b) || !stream(&st))
    return PyLong_FromLong(kElsewhere);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = the_gemv(m, id, k, static_cast<const int32_t*>(kd), x, y, b, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// estimate(model, id, l, h, x, e_out, k_out)
PyObject* estimate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *m = nullptr, *x = nullptr, *e = nullptr, *ko = nullptr, *st = nullptr;
  int id = 0, l = 0, h = 0;
  if (n != 7 || the_estimate == nullptr || !PyLong_Check(a[0]) || !address(a[0], &m) || m == nullptr || !as_int(a[1], &id) || !as_int(a[2], &l) ||
      !as_int(a[3], &h) || !tensor(a[4], &x) || !tensor(a[5], &e) || !tensor(a[6], &ko) || !stream(&st))
    return PyLong_FromLong(kElsewhere);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = the_estimate(m, id, l, h, x, static_cast<float*>(e), static_cast<int32_t*>(ko), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// ---- the calls around the linears ----
struct TokenCalls {
  decltype(&dpllm_rope) rope;
  decltype(&dpllm_tree_attention_workspace_bytes) attention_bytes;
  decltype(&dpllm_tree_attention) attention;
  decltype(&dpllm_verify_workspace_bytes) verify_bytes;
  decltype(&dpllm_verify) verify;
  decltype(&dpllm_cache_append) append;
} to{};
// torch.float16, bfloat16, float32, int32, int64, float64, and torch.empty_like
PyObject *dtypes[6] = {}, *empty_like = nullptr;
enum { kInt32 = 3, kInt64 = 4, kFloat64 = 5 };
PyObject *s_dtype = nullptr, *s_shape = nullptr, *s_stride = nullptr, *s_get_device = nullptr, *s_address = nullptr, *s_batch = nullptr, *s_device = nullptr, *s_new_empty = nullptr, *s_requires_grad = nullptr;

// A reference that is given back.
struct Ref {
  PyObject* o;
  explicit Ref(PyObject* o) : o(o) {}
  ~Ref() { Py_XDECREF(o); }
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
  PyObject* give() {
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};

constexpr int kMaxDim = 5;
struct Tensor {
  void* data;
  int dim, dtype;      // dtype: place in `dtypes`
  int64_t size[kMaxDim], stride[kMaxDim], count;
  bool is(int type, int dims) const { return dtype == type && dim == dims; }
  // whether the last `dims` of its dimensions have no gaps
  bool dense(int dims) const {
    int64_t n = 1;
    for (int i = dim - 1; i >= dim - dims; --i) {
      if (size[i] != 1 && stride[i] != n) return false;
      n *= size[i];
    }
    return true;
  }
};

// What a call is made on: the current device and its stream.
struct Place {
  void* stream;
  int device;
  bool find() { return ::stream(&stream, &device); }
};

// What there is to know of a tensor on the current device that is not empty; false: something is out of the ordinary.
bool look(PyObject* o, const Place& at, Tensor* t) {
  const Ref type(PyObject_GetAttr(o, s_dtype));
  t->dtype = -1;
  for (int i = 0; i < 6; ++i)
    if (type.o != nullptr && type.o == dtypes[i]) t->dtype = i;
  if (t->dtype < 0) return false;
  const Ref device(PyObject_CallMethodNoArgs(o, s_get_device)), shape(PyObject_GetAttr(o, s_shape)), stride(PyObject_CallMethodNoArgs(o, s_stride));
  int index = -1;
  if (device.o == nullptr || !as_int(device.o, &index) || index != at.device || shape.o == nullptr || stride.o == nullptr || !PyTuple_Check(shape.o) || !PyTuple_Check(stride.o)) return false;
  t->dim = (int)PyTuple_GET_SIZE(shape.o);
  if (t->dim > kMaxDim || PyTuple_GET_SIZE(stride.o) != t->dim) return false;
  t->count = 1;
  for (int i = 0; i < t->dim; ++i) {
    t->size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape.o, i));
    t->stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(stride.o, i));
    if (t->size[i] < 1 || t->size[i] > INT32_MAX) return false;
    t->count *= t->size[i];
  }
  return tensor(o, &t->data) && !PyErr_Occurred();
}

// A new tensor that torch has made like t.
bool look_new(PyObject* o, const Tensor& like, Tensor* t) {
  *t = like;
  const Ref stride(PyObject_CallMethodNoArgs(o, s_stride));
  if (stride.o == nullptr || !PyTuple_Check(stride.o) || PyTuple_GET_SIZE(stride.o) != t->dim) return false;
  for (int i = 0; i < t->dim; ++i) t->stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(stride.o, i));
  return tensor(o, &t->data) && !PyErr_Occurred();
}

// A dense tensor of this type and shape (the first dims of a, b, c).
bool look_dense(PyObject* o, const Place& at, int dtype, int dims, int64_t a, int64_t b, int64_t c, void** p) {
  Tensor t;
  if (!look(o, at, &t) || !t.is(dtype, dims) || !t.dense(dims)) return false;
  if (t.size[0] != a || (dims > 1 && t.size[1] != b) || (dims > 2 && t.size[2] != c)) return false;
  *p = t.data;
  return true;
}
// the same, or None
bool look_dense_or_none(PyObject* o, const Place& at, int dtype, int dims, int64_t a, int64_t b, int64_t c, void** p) {
  *p = nullptr;
  return o == Py_None || look_dense(o, at, dtype, dims, a, b, c, p);
}

// [batch][tokens][heads][head_dim], the last without gaps
bool heads_of(const Tensor& t, dpllm_heads* h) {
  if (t.dim != 4 || (t.stride[3] != 1 && t.size[3] != 1)) return false;
  *h = {t.data, t.stride[0], t.stride[1], t.stride[2]};
  return true;
}

PyObject* elsewhere() {
  PyErr_Clear();
  return PyLong_FromLong(kElsewhere);
}

bool as_float(PyObject* o, float* f) {
  const double d = PyFloat_AsDouble(o);
  *f = (float)d;
  return !(d == -1.0 && PyErr_Occurred());
}

// bind_tokens(addresses of the functions of TokenCalls, dtypes, torch.empty_like)
PyObject* bind_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* f[6] = {};
  bool ok = n == 3 && PyTuple_Check(a[0]) && PyTuple_GET_SIZE(a[0]) == 6 && PyTuple_Check(a[1]) && PyTuple_GET_SIZE(a[1]) == 6;
  for (int i = 0; ok && i < 6; ++i) ok = address(PyTuple_GET_ITEM(a[0], i), &f[i]);
  if (!ok) {
    PyErr_SetString(PyExc_TypeError, "bind_tokens(addresses, dtypes, empty_like)");
    return nullptr;
  }
  to = {reinterpret_cast<decltype(to.rope)>(f[0]), reinterpret_cast<decltype(to.attention_bytes)>(f[1]), reinterpret_cast<decltype(to.attention)>(f[2]),
        reinterpret_cast<decltype(to.verify_bytes)>(f[3]), reinterpret_cast<decltype(to.verify)>(f[4]), reinterpret_cast<decltype(to.append)>(f[5])};
  for (int i = 0; i < 6; ++i) Py_XSETREF(dtypes[i], Py_NewRef(PyTuple_GET_ITEM(a[1], i)));
  Py_XSETREF(empty_like, Py_NewRef(a[2]));
  Py_RETURN_NONE;
}

// a new reference to the i-th of a tuple of tensors, or to a lone tensor
PyObject* item(PyObject* o, int i) { return Py_NewRef(PyTuple_Check(o) ? PyTuple_GET_ITEM(o, i) : o); }

// A call with a result: the result on success, else the library's code.
PyObject* answer(int rc, PyObject* result) {
  if (rc == DPLLM_OK) return result;
  Py_DECREF(result);
  return PyLong_FromLong(rc);
}

// A launch may wait for room in the queue: other threads of Python go on meanwhile, as with dpllm_gemv.
template <typename F>
int unlocked(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

// whether a gradient is asked for, which is binding.py's business
bool graded(PyObject* o) {
  const Ref r(PyObject_GetAttr(o, s_requires_grad));
  return r.o != Py_False;
}

// rope(x, positions, freqs, out, scale, layout, inverse)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const int m = n == 7 && PyTuple_Check(a[0]) ? (int)PyTuple_GET_SIZE(a[0]) : 1;
  if (n != 7 || to.rope == nullptr || m < 1 || m > DPLLM_MAX_TENSORS || (a[3] != Py_None && (PyTuple_Check(a[3]) ? (int)PyTuple_GET_SIZE(a[3]) != m : PyTuple_Check(a[0]))))
    return elsewhere();
  Tensor x[DPLLM_MAX_TENSORS], pos, freqs;
  dpllm_heads in[DPLLM_MAX_TENSORS], out[DPLLM_MAX_TENSORS];
  int heads[DPLLM_MAX_TENSORS], layout = 0;
  float scale = 0.f;
  Place place;
  const int inverse = PyObject_IsTrue(a[6]);
  if (!place.find() || !look(a[1], place, &pos) || pos.dtype != kInt32 || pos.dim < 1 || pos.dim > 2 || !pos.dense(pos.dim) || !look(a[2], place, &freqs) || !freqs.is(kFloat64, 1) ||
      !freqs.dense(1) || freqs.size[0] > DPLLM_MAX_HEAD_DIM || !as_float(a[4], &scale) || !as_int(a[5], &layout) || inverse < 0)
    return elsewhere();
  const Ref results(PyTuple_New(m));
  if (results.o == nullptr) return elsewhere();
  for (int i = 0; i < m; ++i) {
    const Ref t(item(a[0], i));
    if (!look(t.o, place, &x[i]) || graded(t.o) || x[i].dtype > 2 || !heads_of(x[i], &in[i]) || x[i].dtype != x[0].dtype || x[i].size[0] != x[0].size[0] ||
        x[i].size[1] != x[0].size[1] || x[i].size[3] != x[0].size[3])
      return elsewhere();
    heads[i] = (int)x[i].size[2];
    PyObject* o = a[3] == Py_None ? PyObject_CallOneArg(empty_like, t.o) : item(a[3], i);
    if (o == nullptr) return elsewhere();
    PyTuple_SET_ITEM(results.o, i, o);
    Tensor y;
    if (!(a[3] == Py_None ? look_new(o, x[i], &y) : look(o, place, &y) && !graded(o)) || y.dtype != x[0].dtype || !heads_of(y, &out[i])) return elsewhere();
    for (int j = 0; j < 4; ++j)
      if (y.size[j] != x[i].size[j]) return elsewhere();
  }
  if (pos.size[pos.dim - 1] != x[0].size[1] || (pos.dim == 2 && pos.size[0] != x[0].size[0])) return elsewhere();
  const int rc = unlocked([&] {
    return to.rope(in, out, heads, m, (int)x[0].size[0], (int)x[0].size[1], (int)x[0].size[3], x[0].dtype, (int)(2 * freqs.size[0]), layout,
                   static_cast<const double*>(freqs.data), scale, static_cast<const int32_t*>(pos.data), pos.dim == 1 ? 0 : x[0].size[1], inverse, place.stream);
  });
  return answer(rc, PyTuple_Check(a[0]) ? Py_NewRef(results.o) : item(results.o, 0));
}

// The dpllm_cache of a Cache object on the current device, and its sequences.
bool cache_of(PyObject* o, const Place& place, const dpllm_cache** c, int* batch) {
  const Ref at(PyObject_GetAttr(o, s_address)), b(PyObject_GetAttr(o, s_batch)), device(PyObject_GetAttr(o, s_device));
  void* p = nullptr;
  int index = -1;
  if (at.o == nullptr || b.o == nullptr || device.o == nullptr || !PyLong_Check(at.o) || !address(at.o, &p) || p == nullptr || !as_int(b.o, batch) ||
      !as_int(device.o, &index) || index != place.device)
    return false;
  *c = static_cast<const dpllm_cache*>(p);
  return true;
}

// A workspace of so many bytes, made by a tensor of elements of `es` bytes (the caller's own is left to the long way); nullptr: something is out of the ordinary.
PyObject* space(PyObject* maker, size_t es, size_t need, void** p) {
  *p = nullptr;
  if (need == 0) return Py_NewRef(Py_None);
  const Ref n(PyLong_FromSize_t((need + es - 1) / es));
  PyObject* o = n.o == nullptr ? nullptr : PyObject_CallMethodOneArg(maker, s_new_empty, n.o);
  if (o != nullptr && tensor(o, p)) return o;
  Py_XDECREF(o);
  return nullptr;
}

// attention(cache, layer, lens, q, k_new, v_new, mask, scale, out, lse, max_len, workspace)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const dpllm_cache* c = nullptr;
  int sequences = 0, layer = 0, max_len = 0;
  Tensor q, k{}, v{}, m{}, y;
  dpllm_heads hq, hk{}, hv{}, ho;
  float scale = 0.f;
  void *lens = nullptr, *lse = nullptr, *ws = nullptr;
  Place place;
  size_t bytes = 0;
  if (n != 12 || to.attention == nullptr || !place.find() || !cache_of(a[0], place, &c, &sequences) || !as_int(a[1], &layer) || !look(a[3], place, &q) || q.dtype != c->dtype || !heads_of(q, &hq) ||
      q.size[3] != c->head_dim || q.size[0] > sequences || !look_dense(a[2], place, kInt32, 1, q.size[0], 0, 0, &lens) || (a[4] == Py_None) != (a[5] == Py_None) ||
      !look_dense_or_none(a[9], place, 2, 3, q.size[0], q.size[1], q.size[2], &lse))
    return elsewhere();
  const int64_t b = q.size[0], t = q.size[1];
  if (a[4] != Py_None) {
    if (!look(a[4], place, &k) || !look(a[5], place, &v) || !heads_of(k, &hk) || !heads_of(v, &hv)) return elsewhere();
    for (const Tensor* x : {&k, &v})
      if (x->dtype != q.dtype || x->size[0] != b || x->size[1] != t || x->size[2] != c->heads || x->size[3] != q.size[3]) return elsewhere();
  }
  if (a[6] != Py_None && (!look(a[6], place, &m) || !m.is(kInt64, 3) || !m.dense(3) || (m.size[0] != 1 && m.size[0] != b) || m.size[1] != t || m.size[2] != (t + 63) / 64))
    return elsewhere();
  const int64_t capacity = (int64_t)c->pages_per_seq * c->page;
  if (a[10] == Py_None ? (max_len = capacity > INT32_MAX ? INT32_MAX : (int)capacity, false) : !as_int(a[10], &max_len)) return elsewhere();
  if (max_len > capacity) max_len = (int)capacity;
  if (a[7] == Py_None ? (scale = (float)(1.0 / __builtin_sqrt((double)q.size[3])), false) : !as_float(a[7], &scale)) return elsewhere();
  if (to.attention_bytes((int)b, (int)t, (int)q.size[2], c->heads, (int)q.size[3], max_len, &bytes) != DPLLM_OK) return elsewhere();
  const Ref result(a[8] == Py_None ? PyObject_CallOneArg(empty_like, a[3]) : Py_NewRef(a[8]));
  if (result.o == nullptr || !(a[8] == Py_None ? look_new(result.o, q, &y) : look(result.o, place, &y)) || y.dtype != q.dtype || !heads_of(y, &ho)) return elsewhere();
  for (int j = 0; j < 4; ++j)
    if (y.size[j] != q.size[j]) return elsewhere();
  const Ref held(a[11] == Py_None ? space(a[3], 2, bytes, &ws) : nullptr);
  if (held.o == nullptr) return elsewhere();
  const int rc = unlocked([&] {
    return to.attention(c, layer, (int)b, (int)t, (int)q.size[2], static_cast<const int32_t*>(lens), max_len, &hq, a[4] == Py_None ? nullptr : &hk,
                        a[5] == Py_None ? nullptr : &hv, static_cast<const uint64_t*>(m.data), a[6] == Py_None || m.size[0] == 1 ? 0 : m.size[1] * m.size[2],
                        scale, &ho, static_cast<float*>(lse), ws, bytes, place.stream);
  });
  return answer(rc, Py_NewRef(result.o));
}

// verify(logits, tokens, uniforms, temperature, parents, draft, siblings), outputs and workspace new
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor x, d{};
  void *tokens = nullptr, *parents = nullptr, *uniforms = nullptr, *temperature = nullptr, *ws = nullptr, *out[3] = {};
  Place place;
  int siblings = 0;
  size_t bytes = 0;
  if (n != 7 || to.verify == nullptr || !place.find() || !look(a[0], place, &x) || x.dtype > 2 || x.dim != 3 || (x.stride[2] != 1 && x.size[2] != 1) ||
      !look_dense(a[1], place, kInt32, 2, x.size[0], x.size[1], 0, &tokens) || !look_dense(a[2], place, 2, 2, x.size[0], x.size[1], 0, &uniforms) ||
      !look_dense(a[3], place, 2, 1, x.size[0], 0, 0, &temperature) || !look_dense_or_none(a[4], place, kInt32, 2, x.size[0], x.size[1], 0, &parents) ||
      !as_int(a[6], &siblings))
    return elsewhere();
  if (a[5] != Py_None) {
    if (!look(a[5], place, &d) || d.dtype != x.dtype || d.dim != 3 || (d.stride[2] != 1 && d.size[2] != 1)) return elsewhere();
    for (int i = 0; i < 3; ++i)
      if (d.size[i] != x.size[i]) return elsewhere();
  }
  if (to.verify_bytes((int)x.size[0], (int)x.size[1], (int)x.size[2], x.dtype, d.data != nullptr, siblings, &bytes) != DPLLM_OK) return elsewhere();
  const Ref batch(PyTuple_GetSlice(Ref(PyObject_GetAttr(a[1], s_shape)).o, 0, 1)), results(PyTuple_New(3));
  if (batch.o == nullptr || results.o == nullptr) return elsewhere();
  for (int i = 0; i < 3; ++i) {
    PyObject* o = i == 0 ? PyObject_CallMethodOneArg(a[1], s_new_empty, batch.o) : PyObject_CallOneArg(empty_like, a[1]);
    if (o == nullptr) return elsewhere();
    PyTuple_SET_ITEM(results.o, i, o);
    if (!tensor(o, &out[i])) return elsewhere();
  }
  const Ref held(space(a[1], 4, bytes, &ws));
  if (held.o == nullptr) return elsewhere();
  const int rc = unlocked([&] {
    return to.verify((int)x.size[0], (int)x.size[1], (int)x.size[2], x.dtype, x.data, x.stride[0], x.stride[1], d.data, d.stride[0], d.stride[1],
                     static_cast<const int32_t*>(tokens), static_cast<const int32_t*>(parents), static_cast<const float*>(uniforms),
                     static_cast<const float*>(temperature), siblings, static_cast<int32_t*>(out[0]), static_cast<int32_t*>(out[1]),
                     static_cast<int32_t*>(out[2]), ws, bytes, place.stream);
  });
  return answer(rc, Py_NewRef(results.o));
}

// append(cache, lens, k_new, v_new, path, count, layer)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const dpllm_cache* c = nullptr;
  int sequences = 0, layer = 0;
  Tensor k, v;
  void *lens = nullptr, *path = nullptr, *count = nullptr;
  Place place;
  if (n != 7 || to.append == nullptr || !place.find() || !cache_of(a[0], place, &c, &sequences) || !look(a[2], place, &k) || !look(a[3], place, &v) || k.dtype != c->dtype || v.dtype != c->dtype ||
      k.dim != v.dim || k.dim < 4 || !as_int(a[6], &layer))
    return elsewhere();
  const int at = k.dim - 4;
  for (int i = 0; i < k.dim; ++i)
    if (k.size[i] != v.size[i]) return elsewhere();
  const int64_t b = k.size[at], t = k.size[at + 1];
  for (const Tensor* x : {&k, &v})
    if (x->stride[at + 3] != 1 && x->size[at + 3] != 1) return elsewhere();
  if (k.size[at + 2] != c->heads || k.size[at + 3] != c->head_dim || b > sequences || !look_dense(a[1], place, kInt32, 1, b, 0, 0, &lens) ||
      !look_dense_or_none(a[4], place, kInt32, 2, b, t, 0, &path) || !look_dense_or_none(a[5], place, kInt32, 1, b, 0, 0, &count))
    return elsewhere();
  const dpllm_heads hk{k.data, k.stride[at], k.stride[at + 1], k.stride[at + 2]}, hv{v.data, v.stride[at], v.stride[at + 1], v.stride[at + 2]};
  const int rc = unlocked([&] {
    return to.append(c, layer, at ? (int)k.size[0] : 1, (int)b, (int)t, static_cast<const int32_t*>(lens), &hk, at ? k.stride[0] : 0, &hv,
                     at ? v.stride[0] : 0, static_cast<const int32_t*>(path), t, static_cast<const int32_t*>(count), place.stream);
  });
  return PyLong_FromLong(rc);
}

using Fast = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyCFunction as_method(Fast f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef methods[] = {{"bind", as_method(bind), METH_FASTCALL, nullptr},
                         {"gemv", as_method(gemv), METH_FASTCALL, nullptr},
                         {"estimate", as_method(estimate), METH_FASTCALL, nullptr},
                         {"bind_tokens", as_method(bind_tokens), METH_FASTCALL, nullptr},
                         {"rope", as_method(rope), METH_FASTCALL, nullptr},
                         {"attention", as_method(attention), METH_FASTCALL, nullptr},
                         {"verify", as_method(verify), METH_FASTCALL, nullptr},
                         {"append", as_method(append), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_dim = PyUnicode_InternFromString("dim");
  s_size = PyUnicode_InternFromString("size");
  zero = PyLong_FromLong(0);
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_address = PyUnicode_InternFromString("address");
  s_batch = PyUnicode_InternFromString("batch");
  s_device = PyUnicode_InternFromString("device");
  s_new_empty = PyUnicode_InternFromString("new_empty");
  s_requires_grad = PyUnicode_InternFromString("requires_grad");
  for (PyObject* s : {s_dtype, s_shape, s_stride, s_get_device, s_address, s_batch, s_device, s_new_empty, s_requires_grad})
    if (s == nullptr) return nullptr;
  if (s_data_ptr == nullptr || s_dim == nullptr || s_size == nullptr || zero == nullptr) return nullptr;
  PyObject* m = PyModule_Create(&definition);
  if (m != nullptr && PyModule_AddIntConstant(m, "ELSEWHERE", kElsewhere) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
