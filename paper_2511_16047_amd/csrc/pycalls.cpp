// The calls that a model makes for every layer and scale -- amskv_append_scale, amskv_attend, amskv_append_scale_rotary,
// amskv_rotate and amskv_cross_attend -- as a CPython extension: argument marshalling only, for binding.py (all other calls
// go through ctypes).  One image through a 16-layer stack is 320 of these calls and 160 short launches, and with ctypes and
// torch's public stream lookup (about 3.6 us a call by itself) the host side took longer than the kernels: 1908 us a pass, 719
// with this (launches included).  The library stays behind its C ABI: bind() and bind_operators() are given the addresses of the
// functions.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <cstdint>

namespace {

typedef int32_t (*Append)(void*, int32_t, int32_t, const void*, const void*, void*);
typedef int32_t (*Attend)(void*, int32_t, int32_t, const void*, void*, void*);
typedef int32_t (*AppendRotary)(void*, int32_t, int32_t, const void*, const void*, const void*, int64_t, void*, void*, const void*, void*);
typedef int32_t (*Rotate)(const void*, int32_t, int32_t, int32_t, int32_t, int32_t, const void*, int64_t, int32_t, const void*, const void*, void*,
                          const void*, void*);
typedef int32_t (*Cross)(const void*, const void*, const void*, const void*, void*, const void*, const void*, void*, uint64_t, void*);
Append append_fn = nullptr;
Attend attend_fn = nullptr;
AppendRotary append_rotary_fn = nullptr;
Rotate rotate_fn = nullptr;
Cross cross_fn = nullptr;
PyObject *rope_class = nullptr, *strides_class = nullptr, *cross_class = nullptr;
PyObject* lookup = nullptr;  // asked once, when a call first leaves the stream to torch: (current device, current stream) functions
PyObject *get_device = nullptr, *get_stream = nullptr;  // its answer; None: there is no device
PyObject *name_data_ptr = nullptr, *name_cuda_stream = nullptr;

bool integer(PyObject* o, int32_t* out) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return false;
  *out = (int32_t)v;
  return true;
}

bool wide(PyObject* o, int64_t* out) {
  *out = PyLong_AsLongLong(o);
  return *out != -1 || !PyErr_Occurred();
}

// None or a structure of the binding's: where it lies (the caller holds it)
bool structure(PyObject* o, PyObject* of, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != of) {
    PyErr_SetString(PyExc_TypeError, "a structure of the binding expected");
    return false;
  }
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return false;
  *out = view.buf;
  PyBuffer_Release(&view);
  return true;
}

bool address(PyObject* o, void** out) {
  *out = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLongMask(o));
  return *out != reinterpret_cast<void*>(UINTPTR_MAX) || !PyErr_Occurred();
}

// None, a device address, or a tensor
bool tensor(PyObject* o, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (PyLong_Check(o)) return address(o, out);
  PyObject* p = PyObject_CallMethodNoArgs(o, name_data_ptr);
  if (!p) return false;
  const bool ok = address(p, out);
  Py_DECREF(p);
  return ok;
}

bool find_stream_functions() {
  PyObject* two = PyObject_CallNoArgs(lookup);
  if (!two) return false;
  PyObject *device, *current;
  const bool ok = PyArg_ParseTuple(two, "OO", &device, &current);
  if (ok) {
    Py_XSETREF(get_device, Py_NewRef(device));
    Py_XSETREF(get_stream, Py_NewRef(current));
  }
  Py_DECREF(two);
  return ok;
}

// None (torch's current stream of the current device), a raw handle, or a stream object
bool stream(PyObject* o, void** out) {
  *out = nullptr;
  if (PyLong_Check(o)) return address(o, out);
  PyObject* p;
  if (o == Py_None) {
    if (!get_stream && !find_stream_functions()) return false;
    if (get_stream == Py_None) return true;
    PyObject* dev = PyObject_CallNoArgs(get_device);
    if (!dev) return false;
    p = PyObject_CallOneArg(get_stream, dev);
    Py_DECREF(dev);
  } else {
    p = PyObject_GetAttr(o, name_cuda_stream);
  }
  if (!p) return false;
  const bool ok = address(p, out);
  Py_DECREF(p);
  return ok;
}

// (cache, layer, s, tensor, tensor, stream) -> status
template <typename F>
PyObject* call(F fn, PyObject* const* args, Py_ssize_t n) {
  int32_t layer, s, status;
  void *cache, *a, *b, *st;
  if (n != 6 || !fn) {
    PyErr_SetString(PyExc_TypeError, "(cache, layer, s, tensor, tensor, stream) expected, after bind()");
    return nullptr;
  }
  if (args[0] == Py_None) cache = nullptr;
  else if (!address(args[0], &cache)) return nullptr;
  if (!integer(args[1], &layer) || !integer(args[2], &s) || !tensor(args[3], &a) || !tensor(args[4], &b) || !stream(args[5], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS  // in the token modes a call may wait for a layer's Eq. 3 test
  status = fn(cache, layer, s, a, b, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

PyObject* append_scale(PyObject*, PyObject* const* args, Py_ssize_t n) { return call(append_fn, args, n); }
PyObject* attend(PyObject*, PyObject* const* args, Py_ssize_t n) { return call(attend_fn, args, n); }

bool handle(PyObject* o, void** out) {
  *out = nullptr;
  return o == Py_None || address(o, out);
}

bool arguments(Py_ssize_t n, Py_ssize_t expected, bool bound) {
  if (n == expected && bound) return true;
  PyErr_SetString(PyExc_TypeError, "the arguments of the C call expected, after bind_operators()");
  return false;
}

// (cache, layer, s, rope, table, Q, q_token_stride, Q_out, K, V, stream) -> status
PyObject* append_scale_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t layer, s, status;
  int64_t q_stride;
  void *cache, *rope, *table, *q, *q_out, *k, *v, *st;
  if (!arguments(n, 11, append_rotary_fn) || !handle(a[0], &cache) || !integer(a[1], &layer) || !integer(a[2], &s) ||
      !structure(a[3], rope_class, &rope) || !tensor(a[4], &table) || !tensor(a[5], &q) || !wide(a[6], &q_stride) || !tensor(a[7], &q_out) ||
      !tensor(a[8], &k) || !tensor(a[9], &v) || !stream(a[10], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  status = append_rotary_fn(cache, layer, s, rope, table, q, q_stride, q_out, k, v, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (rope, dtype, head_dim, batch, heads, tokens, table, table_batch, inverse, x, x strides, out, out strides, stream) -> status
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t size[5], inverse, status;
  int64_t table_batch;
  void *rope, *table, *x, *xs, *out, *os, *st;
  if (!arguments(n, 14, rotate_fn) || !structure(a[0], rope_class, &rope)) return nullptr;
  for (int i = 0; i < 5; ++i)
    if (!integer(a[1 + i], &size[i])) return nullptr;
  if (!tensor(a[6], &table) || !wide(a[7], &table_batch) || !integer(a[8], &inverse) || !tensor(a[9], &x) || !structure(a[10], strides_class, &xs) ||
      !tensor(a[11], &out) || !structure(a[12], strides_class, &os) || !stream(a[13], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  status = rotate_fn(rope, size[0], size[1], size[2], size[3], size[4], table, table_batch, inverse, x, xs, out, os, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (cross, Q, K, V, O, lengths, offsets, workspace, workspace_bytes, stream) -> status
PyObject* cross_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  int32_t status;
  int64_t bytes;
  void *cross, *t[7], *st;
  if (!arguments(n, 10, cross_fn) || !structure(a[0], cross_class, &cross)) return nullptr;
  for (int i = 0; i < 7; ++i)
    if (!tensor(a[1 + i], &t[i])) return nullptr;
  if (!wide(a[8], &bytes) || !stream(a[9], &st)) return nullptr;
  Py_BEGIN_ALLOW_THREADS
  status = cross_fn(cross, t[0], t[1], t[2], t[3], t[4], t[5], t[6], (uint64_t)bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// bind_operators(addresses of amskv_append_scale_rotary, amskv_rotate, amskv_cross_attend, the classes Rope, Strides, Cross)
PyObject* bind_operators(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "six arguments expected");
    return nullptr;
  }
  void *f, *g, *h;
  if (!address(a[0], &f) || !address(a[1], &g) || !address(a[2], &h)) return nullptr;
  append_rotary_fn = reinterpret_cast<AppendRotary>(f);
  rotate_fn = reinterpret_cast<Rotate>(g);
  cross_fn = reinterpret_cast<Cross>(h);
  Py_XSETREF(rope_class, Py_NewRef(a[3]));
  Py_XSETREF(strides_class, Py_NewRef(a[4]));
  Py_XSETREF(cross_class, Py_NewRef(a[5]));
  Py_RETURN_NONE;
}

// bind(address of amskv_append_scale, address of amskv_attend, lookup)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "three arguments expected");
    return nullptr;
  }
  void *f, *g;
  if (!address(args[0], &f) || !address(args[1], &g)) return nullptr;
  append_fn = reinterpret_cast<Append>(f);
  attend_fn = reinterpret_cast<Attend>(g);
  Py_XSETREF(lookup, Py_NewRef(args[2]));
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, "function addresses and stream lookup"},
    {"append_scale", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(append_scale)), METH_FASTCALL, "amskv_append_scale"},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend)), METH_FASTCALL, "amskv_attend"},
    {"append_scale_rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(append_scale_rotary)), METH_FASTCALL, "amskv_append_scale_rotary"},
    {"rotate", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rotate)), METH_FASTCALL, "amskv_rotate"},
    {"cross_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(cross_attend)), METH_FASTCALL, "amskv_cross_attend"},
    {"bind_operators", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind_operators)), METH_FASTCALL, "function addresses and structures"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycalls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pycalls() {
  name_data_ptr = PyUnicode_InternFromString("data_ptr");
  name_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  return name_data_ptr && name_cuda_stream ? PyModule_Create(&module) : nullptr;
}
