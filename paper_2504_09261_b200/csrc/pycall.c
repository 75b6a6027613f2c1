/* Marshalling of the per-step calls from Python, in C: call(address, handle, layer, scale, buffer, ...)
 * calls the entry point at `address` of the C ABI (hack.h) with three to five buffer arguments and
 * returns its status.  A buffer is None, an integer address or an object with a data_ptr() method.
 * The same call through ctypes takes 1.9 us of host time per step against 0.5; a small step keeps the GPU
 * busy for 2 to 3 us, so a caller that enqueues step by step was limited by it. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *data_ptr_name, *dtype_name, *shape_name, *stride_name, *get_device_name;

static int address_of(PyObject* o, void** out) {
  if (o == Py_None) {
    *out = NULL;
    return 0;
  }
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
  }
  PyObject* r = PyObject_CallMethodNoArgs(o, data_ptr_name);
  if (!r) return -1;
  *out = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

static PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n < 7 || n > 9) {
    PyErr_SetString(PyExc_TypeError, "call(address, handle, layer, scale, 3 to 5 buffers)");
    return NULL;
  }
  void* fn = PyLong_AsVoidPtr(args[0]);
  void* h = PyLong_AsVoidPtr(args[1]);
  const long layer = PyLong_AsLong(args[2]), scale = PyLong_AsLong(args[3]);
  void* p[5] = {NULL, NULL, NULL, NULL, NULL};
  if (PyErr_Occurred()) return NULL;
  for (Py_ssize_t i = 4; i < n; ++i)
    if (address_of(args[i], &p[i - 4])) return NULL;
  int status;
  Py_BEGIN_ALLOW_THREADS
  const int32_t l = (int32_t)layer, k = (int32_t)scale;
  if (n == 7) status = ((int (*)(void*, int32_t, int32_t, void*, void*, void*))fn)(h, l, k, p[0], p[1], p[2]);
  else if (n == 8) status = ((int (*)(void*, int32_t, int32_t, void*, void*, void*, void*))fn)(h, l, k, p[0], p[1], p[2], p[3]);
  else status = ((int (*)(void*, int32_t, int32_t, void*, void*, void*, void*, void*))fn)(h, l, k, p[0], p[1], p[2], p[3], p[4]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

/* invoke(address, buffer, ...): an entry point whose arguments are all pointers. */
static PyObject* invoke(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n < 1 || n > 15) {
    PyErr_SetString(PyExc_TypeError, "invoke(address, buffers...)");
    return NULL;
  }
  void* fn = PyLong_AsVoidPtr(args[0]);
  void* p[14] = {NULL};
  if (PyErr_Occurred()) return NULL;
  for (Py_ssize_t i = 1; i < n; ++i)
    if (address_of(args[i], &p[i - 1])) return NULL;
  int status = -1;
#define P0_5 p[0], p[1], p[2], p[3], p[4], p[5]
#define V6 void*, void*, void*, void*, void*, void*
  Py_BEGIN_ALLOW_THREADS
  switch (n - 1) {
    case 6: status = ((int (*)(V6))fn)(P0_5); break;
    case 7: status = ((int (*)(V6, void*))fn)(P0_5, p[6]); break;
    case 8: status = ((int (*)(V6, void*, void*))fn)(P0_5, p[6], p[7]); break;
    case 14: status = ((int (*)(V6, V6, void*, void*))fn)(P0_5, p[6], p[7], p[8], p[9], p[10], p[11], p[12], p[13]); break;
  }
  Py_END_ALLOW_THREADS
#undef P0_5
#undef V6
  if (status < 0) {
    PyErr_SetString(PyExc_TypeError, "invoke: 6, 7, 8 or 14 buffers");
    return NULL;
  }
  return PyLong_FromLong(status);
}

/* key(tensor, ...): of each dtype, shape, strides and device, None for a None; what the arguments of a call that are not addresses
 * depend on.  In C because the same tuple costs a small call as much as its launch (eleven tensors: 9 us; here 4). */
static PyObject* key(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  PyObject* out = PyTuple_New(4 * n);
  if (!out) return NULL;
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* x = args[i];
    PyObject* got[4] = {NULL, NULL, NULL, NULL};
    if (x == Py_None) {
      for (int k = 0; k < 4; ++k) got[k] = Py_NewRef(Py_None);
    } else {
      got[0] = PyObject_GetAttr(x, dtype_name);
      got[1] = got[0] ? PyObject_GetAttr(x, shape_name) : NULL;
      got[2] = got[1] ? PyObject_CallMethodNoArgs(x, stride_name) : NULL;
      got[3] = got[2] ? PyObject_CallMethodNoArgs(x, get_device_name) : NULL;
    }
    for (int k = 0; k < 4; ++k) {
      if (got[k]) { PyTuple_SET_ITEM(out, 4 * i + k, got[k]); continue; }
      Py_DECREF(out);
      return NULL;
    }
  }
  return out;
}

static PyMethodDef methods[] = {{"key", (PyCFunction)(void (*)(void))key, METH_FASTCALL, "key(tensors...) -> tuple"},
                                {"invoke", (PyCFunction)(void (*)(void))invoke, METH_FASTCALL, "invoke(address, buffers...) -> status"},
                                {"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, "call(address, handle, layer, scale, buffers...) -> status"},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hackcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__hackcall(void) {
  data_ptr_name = PyUnicode_InternFromString("data_ptr");
  dtype_name = PyUnicode_InternFromString("dtype");
  shape_name = PyUnicode_InternFromString("shape");
  stride_name = PyUnicode_InternFromString("stride");
  get_device_name = PyUnicode_InternFromString("get_device");
  return data_ptr_name && dtype_name && shape_name && stride_name && get_device_name ? PyModule_Create(&module) : NULL;
}
