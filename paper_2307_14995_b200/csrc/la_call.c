// Python -> C ABI calls without ctypes: call(address, kinds, arg, ...) turns its arguments into those of a C function returning
// la_status, and calls it.
//
// Every argument of the C ABI is an integer or a pointer, so each goes into one 64-bit slot (x86-64 System V: an int is read
// from the slot's low half).  kinds has a letter for each:
//   t  tensor        its address, NULL for None; refused with ValueError unless it is a contiguous CUDA tensor
//   i  integer       its value
//   s  shape         the address of a structure of the type given to bind
//   d  delta shape   the same of the type for the gated delta rule
//   n  norm shape    the same of the type for the norms between two blocks
// Behind a delta shape or a norm shape, tensors of a type and a number of elements that follow from it, on the current device; their gates,
// weights and shared heads make it easy to hand over another one, which would be read out of bounds:
//   Q  q, k          P  dq, dk      (B N Hk d, of in_dtype or out_dtype)
//   V  v, d_o        O  o, dv       (B N H e, likewise)
//   G  fp32, one for each token and value head      S  fp32, a state for each value head
//   X  rows of the residual stream   Y  the other rows   F  fp32, one for each feature
//   w  any tensor on the current device
//   h  host memory   the address of a ctypes array, or the address itself
//   r  stream        what the function given to bind makes of it, asked when the arguments before it have been accepted
// A decode step spends longer in argument conversion than its kernel runs: through ctypes and Python-level checks a call costs
// 5 us before the launch, this way 2.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#define MAX_ARGS 24

static PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_dtype, *s_numel, *s_get_device, *stream_of, *device_of, *dtypes[2];

// include/la.h
typedef struct {
  int B, H, Hk, N, d, e, in_dtype, out_dtype, path, layout;
  float scale;
} DeltaShape;
typedef struct {
  long long rows;
  int D, dtype, res_dtype, gate, post_norm;
  float eps;
} NormShape;
static PyTypeObject *shape_type, *delta_type, *norm_type, *ctypes_array;

// 1: *out holds the slot; 0: an exception is set.
static int slot(char kind, PyObject* a, uint64_t* out) {
  if (kind == 's' || kind == 'd' || kind == 'n' || (kind == 'h' && !PyLong_Check(a))) {
    PyTypeObject* const type = kind == 's' ? shape_type : kind == 'd' ? delta_type : kind == 'n' ? norm_type : ctypes_array;
    if (!type || !PyObject_TypeCheck(a, type)) {
      PyErr_Format(PyExc_TypeError, "%s is expected, not %.100s",
                   kind == 's' ? "a shape" : kind == 'd' ? "a delta shape" : kind == 'n' ? "a block norm shape" : "a ctypes array", Py_TYPE(a)->tp_name);
      return 0;
    }
    Py_buffer view;
    if (PyObject_GetBuffer(a, &view, PyBUF_SIMPLE) != 0) return 0;
    *out = (uint64_t)(uintptr_t)view.buf;
    PyBuffer_Release(&view);  // (the caller holds the object)
    return 1;
  }
  if (kind == 'r') {
    PyObject* const x = stream_of ? PyObject_CallOneArg(stream_of, a) : NULL;
    if (!x) {
      if (!stream_of) PyErr_SetString(PyExc_RuntimeError, "bind has not been called");
      return 0;
    }
    const int ok = slot('i', x, out);
    Py_DECREF(x);
    return ok;
  }
  if (kind != 't') {
    if (!PyLong_Check(a)) {
      PyErr_Format(PyExc_TypeError, "an integer is expected, not %.100s", Py_TYPE(a)->tp_name);
      return 0;
    }
    *out = PyLong_AsUnsignedLongLongMask(a);
    return !(*out == (uint64_t)-1 && PyErr_Occurred());
  }
  if (a == Py_None) {
    *out = 0;
    return 1;
  }
  PyObject* x = PyObject_GetAttr(a, s_is_cuda);
  if (!x) return 0;
  int ok = PyObject_IsTrue(x);
  Py_DECREF(x);
  if (ok > 0) {
    x = PyObject_CallMethodNoArgs(a, s_is_contiguous);
    if (!x) return 0;
    ok = PyObject_IsTrue(x);
    Py_DECREF(x);
  }
  if (ok < 0) return 0;
  if (!ok) {
    PyErr_SetString(PyExc_ValueError, "tensors must be contiguous CUDA tensors");
    return 0;
  }
  x = PyObject_CallMethodNoArgs(a, s_data_ptr);
  if (!x) return 0;
  *out = PyLong_AsUnsignedLongLong(x);
  Py_DECREF(x);
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

// The product of a shape's sizes; -1 where it is more than 63 bits, which the function called refuses by the shape.
static long long product(long long a, long long b) {
  long long x;
  return a < 0 || b < 0 || __builtin_mul_overflow(a, b, &x) ? -1 : x;
}

// The type (0: bf16, 1: fp32; anything else: any) and the number of elements (-1: any) that a letter stands for.
static void expected(char kind, const void* shape, int is_norm, int* dtype, long long* count) {
  *dtype = -1;
  *count = -1;
  if (kind == 'w' || !shape) return;
  if (is_norm) {
    const NormShape* const s = (const NormShape*)shape;
    *dtype = kind == 'X' ? s->res_dtype : kind == 'Y' ? s->dtype : 1;
    *count = kind == 'F' ? s->D : product(s->rows, s->D);
    return;
  }
  const DeltaShape* const s = (const DeltaShape*)shape;
  const long long rows = product(s->B, s->N);
  *dtype = kind == 'Q' || kind == 'V' ? s->in_dtype : kind == 'P' || kind == 'O' ? s->out_dtype : 1;
  *count = kind == 'Q' || kind == 'P' ? product(product(rows, s->Hk), s->d) : kind == 'V' || kind == 'O' ? product(product(rows, s->H), s->e)
         : kind == 'G' ? product(rows, s->H) : product(product(product(s->B, s->H), s->d), s->e);
}

static int as_long(PyObject* x, long long* out) {  // takes the reference
  if (!x) return 0;
  *out = PyLong_AsLongLong(x);
  Py_DECREF(x);
  return !(*out == -1 && PyErr_Occurred());
}

static int checked(char kind, Py_ssize_t index, PyObject* a, const void* shape, int is_norm, long long device, uint64_t* out) {
  *out = 0;
  if (a == Py_None) return 1;
  int dtype;
  long long count, at, n;
  expected(kind, shape, is_norm, &dtype, &count);
  PyObject* x = PyObject_GetAttr(a, s_dtype);
  if (!x) return 0;
  const int typed = dtype < 0 || (dtype <= 1 && x == dtypes[dtype]);
  Py_DECREF(x);
  if (!as_long(PyObject_CallMethodNoArgs(a, s_numel), &n) || !as_long(PyObject_CallMethodNoArgs(a, s_get_device), &at)) return 0;
  if (!typed || (count >= 0 && n != count)) {
    PyErr_Format(PyExc_ValueError, "argument %zd has to be %S with %lld elements", index, dtype == 0 || dtype == 1 ? dtypes[dtype] : Py_None, count);
    return 0;
  }
  if (at != device) {
    PyErr_Format(PyExc_ValueError, "argument %zd has to be on the current CUDA device", index);
    return 0;
  }
  x = PyObject_CallMethodNoArgs(a, s_is_contiguous);
  if (!x) return 0;
  const int ok = PyObject_IsTrue(x);
  Py_DECREF(x);
  if (ok < 0) return 0;
  if (!ok) {
    PyErr_Format(PyExc_ValueError, "argument %zd has to be contiguous", index);
    return 0;
  }
  x = PyObject_CallMethodNoArgs(a, s_data_ptr);
  if (!x) return 0;
  *out = PyLong_AsUnsignedLongLong(x);
  Py_DECREF(x);
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

typedef int (*Fn)(uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t,
                  uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, uint64_t);

// Slots past the callee's arguments are not read.
static PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  Py_ssize_t kinds_n = 0;
  const char* const kinds = n >= 2 && PyUnicode_Check(args[1]) ? PyUnicode_AsUTF8AndSize(args[1], &kinds_n) : NULL;
  if (!kinds || kinds_n != n - 2 || kinds_n > MAX_ARGS) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "call(address, kinds, arg, ...): a letter for each of up to 24 arguments");
    return NULL;
  }
  uint64_t a[MAX_ARGS] = {0}, fn;
  if (!slot('i', args[0], &fn)) return NULL;
  const void* shape = NULL;
  long long device = -2;
  for (Py_ssize_t i = 0; i < kinds_n; ++i) {
    const char kind = kinds[i];
    if (kind == 'w' || (kind >= 'A' && kind <= 'Z')) {
      if (device == -2 && (!device_of || !as_long(PyObject_CallNoArgs(device_of), &device))) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "bind has not been called");
        return NULL;
      }
      if (!checked(kind, i, args[2 + i], shape, kinds[0] == 'n', device, &a[i])) return NULL;
      continue;
    }
    if (!slot(kind, args[2 + i], &a[i])) return NULL;
    if (kind == 'd' || kind == 'n') shape = (const void*)(uintptr_t)a[i];
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = ((Fn)(uintptr_t)fn)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], a[13], a[14], a[15], a[16], a[17],
                           a[18], a[19], a[20], a[21], a[22], a[23]);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

static PyObject* bind(PyObject* self, PyObject* args) {
  (void)self;
  PyObject *type, *f, *delta, *norm, *device, *bf16, *f32;
  if (!PyArg_ParseTuple(args, "O!OO!O!OOO", &PyType_Type, &type, &f, &PyType_Type, &delta, &PyType_Type, &norm, &device, &bf16, &f32)) return NULL;
  Py_INCREF(device);
  Py_XSETREF(device_of, device);
  Py_INCREF(bf16);
  Py_XSETREF(dtypes[0], bf16);
  Py_INCREF(f32);
  Py_XSETREF(dtypes[1], f32);
  Py_INCREF(type);
  Py_XSETREF(shape_type, (PyTypeObject*)type);
  Py_INCREF(delta);
  Py_XSETREF(delta_type, (PyTypeObject*)delta);
  Py_INCREF(norm);
  Py_XSETREF(norm_type, (PyTypeObject*)norm);
  Py_INCREF(f);
  Py_XSETREF(stream_of, f);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, "bind(type of a shape, function that gives a stream's handle, types of a delta shape and of a norm shape, function that gives the current device, torch.bfloat16, torch.float32)"},
                                {"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, "call(address, kinds, arg, ...) -> status"},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_la_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__la_call(void) {
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_numel = PyUnicode_InternFromString("numel");
  s_get_device = PyUnicode_InternFromString("get_device");
  if (!s_is_cuda || !s_is_contiguous || !s_data_ptr || !s_dtype || !s_numel || !s_get_device) return NULL;
  PyObject* const ctypes = PyImport_ImportModule("ctypes");
  if (!ctypes) return NULL;
  ctypes_array = (PyTypeObject*)PyObject_GetAttrString(ctypes, "Array");
  Py_DECREF(ctypes);
  if (!ctypes_array || !PyType_Check((PyObject*)ctypes_array)) return NULL;
  return PyModule_Create(&module);
}
