/* The addresses of the tensors that a call of the operators on logits is given, after checks, for binding.py (a CPython
 * extension; the library itself knows nothing of Python).
 *
 * What a tensor says of itself costs about 60 ns a question in Python, and a call asks about thirty: together a third of a small
 * call.  Here they are read through the C exchange interface that tensor types publish (DLPack 1: an attribute
 * __dlpack_c_exchange_api__ of the type, a capsule of function pointers), which fills in a description that borrows the
 * tensor's sizes.  This file only accepts: where anything is not as it should be, or not of a plain kind, the answer
 * is None and Python looks again, and says what is wrong. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

/* The interface's structures, laid out as DLPack 1 defines them. */
typedef struct {
  void* data;
  int32_t device_type, device_id;
  int32_t ndim;
  uint8_t type_code, type_bits;
  uint16_t type_lanes;
  const int64_t *shape, *strides;
  uint64_t byte_offset;
} Description;
typedef struct {
  uint32_t major, minor;
  const void* older;
  void* allocate;
  void* managed_from;
  void* managed_to;
  int (*describe)(void* tensor, Description* out);
  void* current_stream;
} Exchange;
enum { ON_GPU = 2, PINNED_HOST = 3, MANAGED = 13, INTEGER = 0, FLOATING = 2, BFLOAT = 4 };

static const Exchange* exchange;
static PyTypeObject* tensor_type;

/* setup(capsule, type) -> whether the interface is of a version that this file knows. */
static PyObject* setup(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  if (n != 2 || !PyCapsule_CheckExact(args[0]) || !PyType_Check(args[1])) {
    PyErr_SetString(PyExc_TypeError, "setup(capsule, type)");
    return NULL;
  }
  const Exchange* e = PyCapsule_GetPointer(args[0], PyCapsule_GetName(args[0]));
  if (!e) return NULL;
  if (e->major != 1 || !e->describe) Py_RETURN_FALSE;
  Py_INCREF(args[1]);
  tensor_type = (PyTypeObject*)args[1];
  exchange = e;
  Py_RETURN_TRUE;
}

/* The address of x; with t filled in if it is a tensor (t->data is then not read elsewhere).  0: look again. */
static int address(PyObject* x, unsigned long long* at, Description* t, int* is_tensor) {
  *is_tensor = 0;
  if (x == Py_None) {
    *at = 0;
    return 1;
  }
  if (PyLong_CheckExact(x)) {
    *at = PyLong_AsUnsignedLongLong(x);
    if (*at == (unsigned long long)-1 && PyErr_Occurred()) {
      PyErr_Clear();
      return 0;
    }
    return 1;
  }
  if (Py_TYPE(x) != tensor_type) return 0;
  if (exchange->describe(x, t)) {
    PyErr_Clear();
    return 0;
  }
  *is_tensor = 1;
  *at = (unsigned long long)(uintptr_t)t->data + t->byte_offset;
  return t->device_type == ON_GPU || t->device_type == PINNED_HOST || t->device_type == MANAGED;
}

static int contiguous(const Description* t, int64_t* count) {
  int64_t n = 1;
  for (int i = t->ndim - 1; i >= 0; --i) {
    if (t->shape[i] != 1 && t->strides && t->strides[i] != n && t->shape[i] != 0) return 0;
    n *= t->shape[i];
  }
  *count = n;
  return 1;
}

/* A matrix of rows of `vocab` elements, `stride` apart (0: vocab, which the tensor's own rows then have to be). */
static int matrix(PyObject* x, int64_t rows, int64_t vocab, int64_t dtype, int64_t stride, unsigned long long* at) {
  Description t;
  int is_tensor;
  if (!address(x, at, &t, &is_tensor)) return 0;
  if (!is_tensor || rows <= 0 || vocab <= 0) return 1;
  const int code = dtype == 1 ? BFLOAT : FLOATING, bits = dtype == 2 ? 32 : 16;   /* IRIS_F16, IRIS_BF16, IRIS_F32 */
  if (dtype < 0 || dtype > 2 || t.type_code != code || t.type_bits != bits || t.type_lanes != 1) return 0;
  int64_t count;
  const int whole = contiguous(&t, &count);
  if (whole) {
    if (stride == 0 && rows > 1 && (t.ndim == 0 || (t.ndim > 1 && t.shape[t.ndim - 1] != vocab))) return 0;
  } else {
    if (stride == 0 && rows > 1) return 0;
    if (t.ndim < 1 || (vocab > 1 && t.strides[t.ndim - 1] != 1)) return 0;
    count = 1;
    for (int i = 0; i < t.ndim; ++i) {
      if (t.shape[i] == 0) return 0;
      count += (t.shape[i] - 1) * t.strides[i];
    }
  }
  if (stride == 0) stride = vocab;
  return stride > 0 && stride <= INT64_MAX / 4 / rows && (rows - 1) * stride + vocab <= count;
}

/* A contiguous buffer of at least `count` elements: int64 where they have 8 bytes, fp32 where 4. */
static int buffer(PyObject* x, int64_t size, int64_t count, unsigned long long* at) {
  Description t;
  int is_tensor;
  int64_t has;
  if (!address(x, at, &t, &is_tensor)) return 0;
  if (!is_tensor || count <= 0) return 1;
  return t.type_code == (size == 8 ? INTEGER : FLOATING) && t.type_bits == size * 8 && t.type_lanes == 1 && contiguous(&t, &has) && has >= count;
}

/* addresses(rows, vocab, dtype, logits, row_stride, dlogits, grad_stride, {buffer, element size, elements of a row} ...)
 * -> the addresses of logits, dlogits and the buffers (0 for None), or None: look again. */
static PyObject* addresses(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  unsigned long long at[16];
  long long v[3], stride[2];
  Py_ssize_t i, k = 0;
  if (!exchange || n < 7 || (n - 7) % 3 || (n - 7) / 3 > 14) Py_RETURN_NONE;
  for (i = 0; i < 3; ++i) v[i] = PyLong_AsLongLong(args[i]);
  for (i = 0; i < 2; ++i) stride[i] = PyLong_AsLongLong(args[4 + 2 * i]);
  if (PyErr_Occurred()) goto again;
  if (v[0] > INT32_MAX || v[1] > INT32_MAX) Py_RETURN_NONE;   /* products below stay in 64 bits */
  for (i = 0; i < 2; ++i)
    if (!matrix(args[3 + 2 * i], v[0], v[1], v[2], stride[i], &at[k++])) Py_RETURN_NONE;
  for (i = 7; i < n; i += 3) {
    const long long size = PyLong_AsLongLong(args[i + 1]), each = PyLong_AsLongLong(args[i + 2]);
    if (PyErr_Occurred()) goto again;
    if (each > INT32_MAX || !buffer(args[i], size, v[0] > 0 && each > 0 ? v[0] * each : 0, &at[k++])) Py_RETURN_NONE;
  }
  PyObject* out = PyTuple_New(k);
  if (!out) return NULL;
  for (i = 0; i < k; ++i) {
    PyObject* a = PyLong_FromUnsignedLongLong(at[i]);
    if (!a) {
      Py_DECREF(out);
      return NULL;
    }
    PyTuple_SET_ITEM(out, i, a);
  }
  return out;
again:
  PyErr_Clear();
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, "setup(capsule, type) -> bool"},
    {"addresses", (PyCFunction)(void (*)(void))addresses, METH_FASTCALL, "addresses of checked tensors, or None"},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&module); }
