/* Marshalling of the per-step calls from Python, in C (run, of the operators around them: further down): call(address, handle, layer, scale, buffer, ...)
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

/* What the arguments of a call that are not addresses depend on: of each tensor dtype, shape, strides and device, None for a None. */
static PyObject* key_of(PyObject* head, PyObject* const* tensors, Py_ssize_t n) {
  PyObject* key = PyTuple_New(1 + 4 * n);
  if (!key) return NULL;
  PyTuple_SET_ITEM(key, 0, Py_NewRef(head));
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *x = tensors[i], *got[4] = {NULL, NULL, NULL, NULL};
    if (x == Py_None) {
      for (int k = 0; k < 4; ++k) got[k] = Py_NewRef(Py_None);
    } else {
      got[0] = PyObject_GetAttr(x, dtype_name);
      got[1] = got[0] ? PyObject_GetAttr(x, shape_name) : NULL;
      got[2] = got[1] ? PyObject_CallMethodNoArgs(x, stride_name) : NULL;
      got[3] = got[2] ? PyObject_CallMethodNoArgs(x, get_device_name) : NULL;
    }
    if (!got[3]) {
      for (int k = 0; k < 3; ++k) Py_XDECREF(got[k]);
      Py_DECREF(key);
      return NULL;
    }
    for (int k = 0; k < 4; ++k) PyTuple_SET_ITEM(key, 1 + 4 * i + k, got[k]);
  }
  return key;
}

/* run(store, head, address, lead, stream, tensor, ...): the entry point at `address` with a lead pointer (a plan, a 4-bit cache), an
 * argument struct, the tensors and the stream.  `store` maps keys (head, which is hashable, and what key_of says of the
 * tensors) to (struct, its address).  Returns the entry point's status, or, where the store has no struct yet, the key. */
static PyObject* run(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  const Py_ssize_t tensors = n - 5;
  if (tensors < 3 || tensors > 11 || !PyDict_Check(args[0])) {
    PyErr_SetString(PyExc_TypeError, "run(store, head, address, lead, stream, tensors...)");
    return NULL;
  }
  void *p[14] = {NULL}, *fn = PyLong_AsVoidPtr(args[2]);
  if (PyErr_Occurred() || address_of(args[3], &p[0])) return NULL;
  PyObject* key = key_of(args[1], args + 5, tensors);
  if (!key) return NULL;
  PyObject* entry = PyDict_GetItemWithError(args[0], key);
  if (!entry) {
    if (!PyErr_Occurred()) return key;
    Py_DECREF(key);
    return NULL;
  }
  Py_INCREF(entry);                            /* (the struct lives on, whatever another thread does to the store) */
  Py_DECREF(key);
  p[1] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(entry, 1));
  int bad = PyErr_Occurred() != NULL;
  for (Py_ssize_t i = 0; i < tensors && !bad; ++i) bad = address_of(args[5 + i], &p[2 + i]);
  if (!bad) bad = address_of(args[4], &p[2 + tensors]);
  int status = -1;
  if (!bad) {
#define P0_5 p[0], p[1], p[2], p[3], p[4], p[5]
#define V6 void*, void*, void*, void*, void*, void*
    Py_BEGIN_ALLOW_THREADS
    switch (tensors + 3) {
      case 6: status = ((int (*)(V6))fn)(P0_5); break;
      case 7: status = ((int (*)(V6, void*))fn)(P0_5, p[6]); break;
      case 8: status = ((int (*)(V6, void*, void*))fn)(P0_5, p[6], p[7]); break;
      case 14: status = ((int (*)(V6, V6, void*, void*))fn)(P0_5, p[6], p[7], p[8], p[9], p[10], p[11], p[12], p[13]); break;
    }
    Py_END_ALLOW_THREADS
#undef P0_5
#undef V6
  }
  Py_DECREF(entry);
  if (bad) return NULL;
  if (status < 0) {
    PyErr_SetString(PyExc_TypeError, "run: 3, 4, 5 or 11 tensors");
    return NULL;
  }
  return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {{"run", (PyCFunction)(void (*)(void))run, METH_FASTCALL, "run(store, head, address, lead, stream, tensors...) -> status or key"},
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
