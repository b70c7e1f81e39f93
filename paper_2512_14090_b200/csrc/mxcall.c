/* CPython entry to the microscaled calls.
 *
 * A small call of these (2 to 5 us on the GPU) spends more time on its way there.  ctypes converts every argument on its own, 80 ns each;
 * this module takes the same plain integers (None = NULL) in the same order and returns the same status: one row through a
 * 1280 x 320 layer 6.8 -> 5.4 us a call, a linear layer of two launches 10.2 -> 8.7.  The binding uses ctypes where it is not built.  No arithmetic and no checks here. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/aiq.h"

/* the arguments as 64-bit integers; 0 with a Python error set if one is neither an integer nor None, or their number is wrong */
static int take(const char* name, PyObject* const* args, Py_ssize_t n, Py_ssize_t want, long long* v) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%s: %zd arguments, not %zd", name, want, n);
    return 0;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (args[i] == Py_None) { v[i] = 0; continue; }
    v[i] = PyLong_AsLongLong(args[i]);
    if (v[i] == -1 && PyErr_Occurred()) return 0;
  }
  return 1;
}
/* an `int` parameter: out of its range, the smallest int, which every entry point refuses */
static int narrow(long long v) { return v < INT_MIN || v > INT_MAX ? INT_MIN : (int)v; }
#define PTR(i) ((void*)(intptr_t)v[i])
#define INT(i) narrow(v[i])

static PyObject* quantize(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  long long v[8];
  int status;
  (void)self;
  if (!take("aiq_mx_quantize", args, n, 8, v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = aiq_mx_quantize(PTR(0), INT(1), INT(2), INT(3), v[4], PTR(5), PTR(6), PTR(7));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

static PyObject* dequantize(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  long long v[8];
  int status;
  (void)self;
  if (!take("aiq_mx_dequantize", args, n, 8, v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = aiq_mx_dequantize(PTR(0), PTR(1), INT(2), INT(3), INT(4), PTR(5), v[6], PTR(7));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

static PyObject* linear(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  long long v[14];
  int status;
  (void)self;
  if (!take("aiq_mx_linear", args, n, 14, v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = aiq_mx_linear(PTR(0), PTR(1), (const float*)PTR(2), INT(3), INT(4), PTR(5), INT(6), INT(7), v[8], PTR(9), v[10], PTR(11),
                         (size_t)v[12], PTR(13));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

static PyObject* matmul(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  long long v[12];
  int status;
  (void)self;
  if (!take("aiq_mx_matmul", args, n, 12, v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = aiq_mx_matmul(PTR(0), PTR(1), INT(2), PTR(3), PTR(4), INT(5), (const float*)PTR(6), INT(7), PTR(8), INT(9), v[10], PTR(11));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {
    {"aiq_mx_quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, NULL},
    {"aiq_mx_dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL, NULL},
    {"aiq_mx_linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, NULL},
    {"aiq_mx_matmul", (PyCFunction)(void (*)(void))matmul, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mxcall", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__mxcall(void) { return PyModule_Create(&module); }
