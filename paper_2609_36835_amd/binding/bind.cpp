// The short way from tensors to the C ABI for calls that a decode step makes: checks of arguments and the call in native
// code, 0.3 us where the same checks in Python take four.  Every function here takes what its namesake in arckv.py takes,
// behind the current device, and returns None for anything that it does not find as documented, or that the library
// refuses: arckv.py then goes the long way, whose errors say what is wrong.  Nothing is computed here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "arckv.h"

namespace {

// Set by init(): entry points of the loaded library, and torch's function from a device to its current stream.
decltype(&arckv_ncache_write) ncache_write_;
decltype(&arckv_ncache_read) ncache_read_;
decltype(&arckv_attend_ncache_workspace_size) attend_ncache_workspace_size_;
decltype(&arckv_attend_ncache) attend_ncache_;
decltype(&arckv_rotary) rotary_;
PyObject *stream_of_;

PyObject *long_way() { Py_RETURN_NONE; }

// The interpreter's lock is open while one of these lives: a launch may wait for room in a queue, an allocation for the GPU.
struct Unlocked {
  PyThreadState *state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F> auto unlocked(F f) {
  Unlocked u;
  return f();
}

// The current device's tensor behind an argument; null for anything else.
const at::Tensor *tensor(PyObject *o, int64_t dev) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  return t.is_cuda() && t.layout() == at::kStrided && t.get_device() == dev ? &t : nullptr;
}

// Pointer of a contiguous tensor of this shape and type; false where the argument is something else.
bool pointer(PyObject *o, int64_t dev, at::ScalarType type, at::IntArrayRef shape, void **p) {
  const at::Tensor *t = tensor(o, dev);
  if (!t || t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) return false;
  *p = t->data_ptr();
  return true;
}
bool pointer_or_none(PyObject *o, int64_t dev, at::ScalarType type, at::IntArrayRef shape, void **p) {
  *p = nullptr;
  return o == Py_None || pointer(o, dev, type, shape, p);
}

bool stream(PyObject *dev, hipStream_t *s) {
  PyObject *r = PyObject_CallOneArg(stream_of_, dev);
  if (!r) return false;
  *s = reinterpret_cast<hipStream_t>(PyLong_AsVoidPtr(r));
  Py_DECREF(r);
  return !PyErr_Occurred();
}

bool cache(PyObject *o, int64_t dev, arckv_ncache *c) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
  const at::Tensor *K = tensor(PyTuple_GET_ITEM(o, 0), dev);
  if (!K || K->dim() != 3) return false;
  const int64_t P = K->size(0), rows = K->size(1);
  if (P > INT32_MAX || rows > INT32_MAX) return false;
  *c = arckv_ncache{(int32_t)P, (int32_t)rows, 128, nullptr, nullptr, nullptr, nullptr};
  return pointer(PyTuple_GET_ITEM(o, 0), dev, at::kByte, {P, rows, 64}, &c->K) &&
         pointer(PyTuple_GET_ITEM(o, 1), dev, at::kByte, {P, rows, 64}, &c->V) &&
         pointer(PyTuple_GET_ITEM(o, 2), dev, at::kByte, {P, rows, 4}, &c->K_scale) &&
         pointer(PyTuple_GET_ITEM(o, 3), dev, at::kByte, {P, rows, 4}, &c->V_scale);
}

bool dtype_of(at::ScalarType t, int32_t *dtype) {
  if (t != at::kBFloat16 && t != at::kFloat) return false;
  *dtype = t == at::kFloat ? ARCKV_F32 : ARCKV_BF16;
  return true;
}

// A number that 32 bits hold, from a plain int.
bool int32_of(PyObject *o, int32_t *x) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow || v < INT32_MIN || v > INT32_MAX) return false;
  *x = (int32_t)v;
  return true;
}

// (device, cache, K, V, start, count)
PyObject *ncache_write(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6) return long_way();
  const int64_t dev = PyLong_AsLongLong(a[0]);
  arckv_ncache c;
  const at::Tensor *K;
  int32_t dtype;
  void *k, *v, *start, *count;
  if (!cache(a[1], dev, &c) || !(K = tensor(a[2], dev)) || K->dim() != 3 || K->size(1) > c.rows ||
      !dtype_of(K->scalar_type(), &dtype))
    return long_way();
  const int64_t rows = K->size(1);
  hipStream_t s;
  if (!pointer(a[2], dev, K->scalar_type(), {c.P, rows, 128}, &k) || !pointer(a[3], dev, K->scalar_type(), {c.P, rows, 128}, &v) ||
      !pointer_or_none(a[4], dev, at::kInt, {c.P}, &start) || !pointer_or_none(a[5], dev, at::kInt, {c.P}, &count))
    return long_way();
  if (!stream(a[0], &s)) return nullptr;
  if (unlocked([&] { return ncache_write_(&c, (int32_t)rows, dtype, k, v, (const int32_t *)start, (const int32_t *)count, s); }) !=
      ARCKV_OK)
    return long_way();
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// (device, cache, first, rows, float32?, length)
PyObject *ncache_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6) return long_way();
  const int64_t dev = PyLong_AsLongLong(a[0]);
  arckv_ncache c;
  int32_t first, rows;
  void *length;
  if (!cache(a[1], dev, &c) || !int32_of(a[2], &first)) return long_way();
  if (a[3] == Py_None)
    rows = first >= 0 && first < c.rows ? c.rows - first : 0;
  else if (!int32_of(a[3], &rows))
    return long_way();
  if (first < 0 || rows < 1 || rows > c.rows || first > c.rows - rows || !pointer_or_none(a[5], dev, at::kInt, {c.P}, &length))
    return long_way();
  const at::ScalarType type = a[4] == Py_True ? at::kFloat : at::kBFloat16;
  hipStream_t s;
  if (!stream(a[0], &s)) return nullptr;
  const auto options = THPVariable_Unpack(PyTuple_GET_ITEM(a[1], 0)).options().dtype(type);
  at::Tensor K, V;
  const arckv_status got = unlocked([&] {
    K = at::empty({c.P, rows, 128}, options);
    V = at::empty({c.P, rows, 128}, options);
    return ncache_read_(&c, first, rows, type == at::kFloat ? ARCKV_F32 : ARCKV_BF16, (const int32_t *)length, K.data_ptr(),
                        V.data_ptr(), s);
  });
  if (got != ARCKV_OK) return long_way();
  PyObject *k = THPVariable_Wrap(std::move(K)), *v = THPVariable_Wrap(std::move(V));
  PyObject *both = k && v ? PyTuple_Pack(2, k, v) : nullptr;
  Py_XDECREF(k);
  Py_XDECREF(v);
  return both;
  END_HANDLE_TH_ERRORS
}

// (device, Q, cache, beta, length, K_f, V_f, length_f, scale, out, ws)
PyObject *attend_ncache(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11) return long_way();
  const int64_t dev = PyLong_AsLongLong(a[0]);
  arckv_ncache c;
  const at::Tensor *Q, *Kf = nullptr, *ws = nullptr;
  void *q, *beta, *length, *kf, *vf, *length_f, *w = nullptr;
  if (!cache(a[2], dev, &c) || !(Q = tensor(a[1], dev)) || Q->dim() != 3 || Q->size(1) > INT32_MAX) return long_way();
  const int64_t G = Q->size(1);
  if (a[5] != Py_None && (!(Kf = tensor(a[5], dev)) || Kf->dim() != 3 || Kf->size(1) > INT32_MAX)) return long_way();
  const int64_t F = Kf ? Kf->size(1) : 0;
  if (!pointer(a[1], dev, at::kBFloat16, {c.P, G, 128}, &q) || !pointer_or_none(a[3], dev, at::kFloat, {c.P, c.rows}, &beta) ||
      !pointer_or_none(a[4], dev, at::kInt, {c.P}, &length) || !pointer_or_none(a[5], dev, at::kBFloat16, {c.P, F, 128}, &kf) ||
      !pointer_or_none(a[6], dev, at::kBFloat16, {c.P, F, 128}, &vf) || !pointer_or_none(a[7], dev, at::kInt, {c.P}, &length_f))
    return long_way();
  double scale = 0.0;
  if (a[8] != Py_None) {
    if (!PyFloat_CheckExact(a[8])) return long_way();
    scale = PyFloat_AS_DOUBLE(a[8]);
  }
  size_t bytes = 0;
  if (a[10] == Py_None) {
    if (attend_ncache_workspace_size_(c.P, c.rows, (int32_t)G, (int32_t)F, &bytes) != ARCKV_OK) return long_way();
  } else {
    if (!(ws = tensor(a[10], dev)) || ws->scalar_type() != at::kByte || !ws->is_contiguous()) return long_way();
    bytes = (size_t)ws->numel();
    w = ws->data_ptr();
  }
  void *o;
  if (a[9] != Py_None && !pointer(a[9], dev, at::kFloat, {c.P, G, 128}, &o)) return long_way();
  hipStream_t s;
  if (!stream(a[0], &s)) return nullptr;
  at::Tensor out;
  const bool new_out = a[9] == Py_None;
  const arckv_status got = unlocked([&] {
    at::Tensor space;
    if (new_out) {
      out = at::empty({c.P, G, 128}, Q->options().dtype(at::kFloat));
      o = out.data_ptr();
    }
    if (!w && bytes) {   // torch's device allocations are 512-byte aligned
      space = at::empty({(int64_t)bytes}, Q->options().dtype(at::kByte));
      w = space.data_ptr();
    }
    return attend_ncache_(&c, (int32_t)G, (int32_t)F, (float)scale, q, (const float *)beta, (const int32_t *)length, kf, vf,
                          (const int32_t *)length_f, (float *)o, w, bytes, s);
  });
  if (got != ARCKV_OK) return long_way();
  if (a[9] == Py_None) return THPVariable_Wrap(std::move(out));
  Py_INCREF(a[9]);
  return a[9];
  END_HANDLE_TH_ERRORS
}

bool rows_of(PyObject *x, PyObject *y, int64_t dev, int64_t N, at::ScalarType type, arckv_rotary_rows *r) {
  const at::Tensor *u = tensor(x, dev), *v = tensor(y, dev);
  if (!u || !v || u->scalar_type() != type || v->scalar_type() != type || u->dim() != 3 || u->size(0) != N || u->size(2) != 128 ||
      v->sizes() != u->sizes() || u->stride(2) != 1 || v->stride(2) != 1 || u->size(1) > INT32_MAX)
    return false;
  const int64_t heads = u->size(1);   // the stride of an axis of one says nothing
  *r = arckv_rotary_rows{(int32_t)heads, u->data_ptr(), N == 1 ? 0 : u->stride(0), heads == 1 ? 0 : u->stride(1),
                         v->data_ptr(), N == 1 ? 0 : v->stride(0), heads == 1 ? 0 : v->stride(1)};
  return true;
}

// (device, x, freq, positions, other, interleaved, transpose, factor, out, out_other): outputs are given
PyObject *rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10) return long_way();
  const int64_t dev = PyLong_AsLongLong(a[0]);
  const at::Tensor *x = tensor(a[1], dev), *f = tensor(a[2], dev);
  arckv_rotary_rows r[2];
  int32_t dtype;
  void *freq, *positions;
  if (!x || !f || x->dim() != 3 || x->size(0) > INT32_MAX || f->dim() != 1 || f->size(0) > 64 || !dtype_of(x->scalar_type(), &dtype) ||
      !PyBool_Check(a[5]) || !PyBool_Check(a[6]) || !PyFloat_CheckExact(a[7]))
    return long_way();
  const int64_t N = x->size(0), pairs = f->size(0);
  if (!pointer(a[2], dev, at::kDouble, {pairs}, &freq) || !pointer_or_none(a[3], dev, at::kInt, {N}, &positions) ||
      !rows_of(a[1], a[8], dev, N, x->scalar_type(), &r[0]) ||
      (a[4] != Py_None && !rows_of(a[4], a[9], dev, N, x->scalar_type(), &r[1])))
    return long_way();
  const arckv_rotary_params p = {(int32_t)N, 128, 2 * (int32_t)pairs, a[5] == Py_True ? ARCKV_ROTARY_NEIGHBOURS : ARCKV_ROTARY_HALVES,
                                 dtype, a[6] == Py_True, (float)PyFloat_AS_DOUBLE(a[7])};
  hipStream_t s;
  if (!stream(a[0], &s)) return nullptr;
  const arckv_rotary_rows *other = a[4] != Py_None ? &r[1] : nullptr;
  if (unlocked([&] { return rotary_(&p, (const int32_t *)positions, (const double *)freq, &r[0], other, s); }) != ARCKV_OK)
    return long_way();
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// init(addresses of the entry points in the order above, the function from a device to its stream)
PyObject *init(PyObject *, PyObject *args) {
  unsigned long long p[5];
  PyObject *f;
  if (!PyArg_ParseTuple(args, "(KKKKK)O", &p[0], &p[1], &p[2], &p[3], &p[4], &f)) return nullptr;
  ncache_write_ = reinterpret_cast<decltype(ncache_write_)>(p[0]);
  ncache_read_ = reinterpret_cast<decltype(ncache_read_)>(p[1]);
  attend_ncache_workspace_size_ = reinterpret_cast<decltype(attend_ncache_workspace_size_)>(p[2]);
  attend_ncache_ = reinterpret_cast<decltype(attend_ncache_)>(p[3]);
  rotary_ = reinterpret_cast<decltype(rotary_)>(p[4]);
  Py_INCREF(f);
  Py_XSETREF(stream_of_, f);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr},
                         {"ncache_write", (PyCFunction)(void (*)(void))ncache_write, METH_FASTCALL, nullptr},
                         {"ncache_read", (PyCFunction)(void (*)(void))ncache_read, METH_FASTCALL, nullptr},
                         {"attend_ncache", (PyCFunction)(void (*)(void))attend_ncache, METH_FASTCALL, nullptr},
                         {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_arckv_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch whose C++ types this file was compiled with; used with another it may read them wrongly.
PyMODINIT_FUNC PyInit__arckv_bind() {
  PyObject *m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", ARCKV_TORCH) < 0) Py_CLEAR(m);
  return m;
}
