/* Argument marshalling of the calls that run once per layer and step (rms_norm, route, AdapterBank.forward), as a CPython
 * extension: checks of the tensors' types, devices, shapes and strides, the current stream, and the call into the C ABI.  The same in
 * Python and ctypes takes 10 us of host time per call, longer than the kernels of a decode step.  No torch headers: tensors are
 * asked through their Python attributes.  The functions of the library come in as addresses (init). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/swapmoe.h"

typedef int32_t (*rms_norm_fn)(const swapmoe_rms_norm_t*, void*);
typedef int32_t (*route_fn)(const swapmoe_gate_t*, const float*, int64_t, const float*, const int32_t*, int32_t, int32_t, int32_t,
                            int32_t*, float*, int32_t*, void*);
typedef int32_t (*adapters_fn)(swapmoe_adapters_t*, const void*, int64_t, const float*, const int32_t*, const void*, int64_t, void*,
                               int64_t, int32_t, void*);

static rms_norm_fn f_rms_norm;
static route_fn f_route;
static adapters_fn f_adapters;
static PyObject *fail, *d_f32, *d_bf16, *d_e4m3, *d_i32;                      /* the error function, torch's types */
static PyObject *get_device_fn, *set_device_fn, *raw_stream_fn;               /* torch's current device and stream */
static PyObject *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_get_device, *s_is_contiguous, *s_cuda_stream, *s_numel;

typedef struct {
  const char* where;
  long device;               /* -1: not known yet */
} Call;

/* Raises the package's error with `status` and a text. */
static int refuse(const Call* c, int status, const char* format, ...) {
  va_list v;
  va_start(v, format);
  PyObject* text = PyUnicode_FromFormatV(format, v);
  va_end(v);
  if (text) {
    PyObject* r = PyObject_CallFunction(fail, "isO", status, c->where, text);
    Py_XDECREF(r);
    Py_DECREF(text);
    if (r) PyErr_SetString(PyExc_RuntimeError, c->where);
  }
  return -1;
}

/* A tensor's device (the first one's has to be a GPU, the others' the same) and address. */
static int place(Call* c, PyObject* t, const char* name, void** p) {
  PyObject* v = PyObject_CallMethodNoArgs(t, s_get_device);
  if (!v) return -1;
  const long dev = PyLong_AsLong(v);
  Py_DECREF(v);
  if (dev == -1 && PyErr_Occurred()) return -1;
  if (dev < 0) return refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: a CUDA tensor expected", name);
  if (c->device < 0) c->device = dev;
  if (c->device != dev) return refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: on device %ld, the others on %ld", name, dev, c->device);
  v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!v) return -1;
  *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return PyErr_Occurred() ? -1 : 0;
}

static int type_is(Call* c, PyObject* t, const char* name, PyObject* dtype) {
  PyObject* v = PyObject_GetAttr(t, s_dtype);
  if (!v) return -1;
  const int same = v == dtype;
  if (!same) refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: %S expected, got %S", name, dtype, v);
  Py_DECREF(v);
  return same ? 0 : -1;
}

/* SWAPMOE_F32 or SWAPMOE_BF16 of a tensor's type. */
static int layer_type(Call* c, PyObject* t, const char* name, int32_t* dtype, PyObject** object) {
  PyObject* v = PyObject_GetAttr(t, s_dtype);
  if (!v) return -1;
  Py_DECREF(v);                                     /* (torch keeps its types) */
  *object = v;
  if (v == d_f32) *dtype = SWAPMOE_F32;
  else if (v == d_bf16) *dtype = SWAPMOE_BF16;
  else return refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: float32 or bfloat16 expected, got %S", name, v);
  return 0;
}

/* Shape of a tensor of one or two dimensions, and the strides. */
static int sizes(Call* c, PyObject* t, const char* name, int* dims, int64_t size[2], int64_t stride[2]) {
  PyObject *a = PyObject_GetAttr(t, s_shape), *b = a ? PyObject_CallMethodNoArgs(t, s_stride) : NULL;
  int rc = -1;
  if (!b) goto done;
  if (!PyTuple_Check(a) || !PyTuple_Check(b) || PyTuple_GET_SIZE(a) != PyTuple_GET_SIZE(b) || PyTuple_GET_SIZE(a) < 1 ||
      PyTuple_GET_SIZE(a) > 2) {
    refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: rows [n, width] expected, got shape %S", name, a);
    goto done;
  }
  *dims = (int)PyTuple_GET_SIZE(a);
  for (int i = 0; i < *dims; ++i) {
    size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(a, i));
    stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(b, i));
  }
  if (size[0] > INT32_MAX || (*dims == 2 && size[1] > INT32_MAX)) {
    refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: too large: %S", name, a);
    goto done;
  }
  rc = PyErr_Occurred() ? -1 : 0;
done:
  Py_XDECREF(a);
  Py_XDECREF(b);
  return rc;
}

/* At least n_rows rows of `width` contiguous values of `dtype`; a vector stands for rows of one value. */
static int rows(Call* c, PyObject* t, const char* name, PyObject* dtype, int64_t n_rows, int64_t width, void** p, int64_t* row_stride) {
  int dims;
  int64_t size[2], stride[2];
  if (type_is(c, t, name, dtype) || sizes(c, t, name, &dims, size, stride) || place(c, t, name, p)) return -1;
  if (dims == 1) { size[1] = 1; stride[1] = 1; }
  if ((dims == 1 && width != 1) || size[0] < n_rows || size[1] != width || (width > 1 && stride[1] != 1))
    return refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: [%lld, %lld] with contiguous rows expected, got [%lld, %lld], strides (%lld, %lld)",
                  name, (long long)n_rows, (long long)width, (long long)size[0], (long long)size[1], (long long)stride[0],
                  (long long)stride[1]);
  *row_stride = size[0] > 1 || stride[0] > width ? stride[0] : width;
  return 0;
}

/* n contiguous values of `dtype`. */
static int vector(Call* c, PyObject* t, const char* name, PyObject* dtype, int64_t n, void** p) {
  if (type_is(c, t, name, dtype) || place(c, t, name, p)) return -1;
  PyObject *a = PyObject_CallMethodNoArgs(t, s_numel), *b = a ? PyObject_CallMethodNoArgs(t, s_is_contiguous) : NULL;
  int rc = -1;
  if (b) {
    const int64_t have = PyLong_AsLongLong(a);
    if (have != n || b != Py_True)
      refuse(c, SWAPMOE_ERR_INVALID_ARG, "%s: %lld contiguous values expected, got %lld%s", name, (long long)n, (long long)have,
             b == Py_True ? "" : ", not contiguous");
    else rc = 0;
  }
  Py_XDECREF(a);
  Py_XDECREF(b);
  return rc;
}

static int integer(PyObject* v, int64_t* out) {
  *out = PyLong_AsLongLong(v);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

/* The stream of a call (an integer, an object with cuda_stream, or None: the device's current one); makes the tensors' device
 * current: *back is the device to return to, or -1. */
static int begin(const Call* c, PyObject* stream, void** st, long* back) {
  PyObject* v;
  *back = -1;
  if (stream == Py_None) {
    PyObject* d = PyLong_FromLong(c->device);
    v = d ? PyObject_CallOneArg(raw_stream_fn, d) : NULL;
    Py_XDECREF(d);
  } else if (PyLong_Check(stream)) {
    v = Py_NewRef(stream);
  } else {
    v = PyObject_GetAttr(stream, s_cuda_stream);
  }
  if (!v) return -1;
  *st = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) return -1;
  v = PyObject_CallNoArgs(get_device_fn);
  if (!v) return -1;
  const long now = PyLong_AsLong(v);
  Py_DECREF(v);
  if (now != c->device) {
    v = PyObject_CallFunction(set_device_fn, "l", c->device);
    if (!v) return -1;
    Py_DECREF(v);
    *back = now;
  }
  return 0;
}

static PyObject* end(const Call* c, long back, int32_t status) {
  if (back >= 0) {
    PyObject* v = PyObject_CallFunction(set_device_fn, "l", back);
    if (!v) return NULL;
    Py_DECREF(v);
  }
  if (status != SWAPMOE_OK) {
    PyObject* r = PyObject_CallFunction(fail, "isO", (int)status, c->where, Py_None);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, c->where);
    return NULL;
  }
  Py_RETURN_NONE;
}

/* rms_norm(x, weight, eps, out, residual, residual_out, out8, scales, group, stream) */
static PyObject* py_rms_norm(PyObject* self, PyObject* const* v, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "ten arguments expected");
  Call c = {"swapmoe_rms_norm", -1};
  swapmoe_rms_norm_t a = {0};
  PyObject *x = v[0], *weight = v[1], *out = v[3], *residual = v[4], *residual_out = v[5], *out8 = v[6], *scales = v[7];
  PyObject *dtype, *rdtype = NULL;
  int dims;
  int64_t size[2], stride[2], group;
  if (layer_type(&c, x, "x", &a.dtype, &dtype) || sizes(&c, x, "x", &dims, size, stride)) return NULL;
  if (dims != 2) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "x: [T, d] expected"); return NULL; }
  const int64_t T = size[0], d = size[1];
  if (integer(v[8], &group)) return NULL;
  if (group < 0 || group > INT32_MAX) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "group: %lld", (long long)group); return NULL; }
  const double eps = PyFloat_AsDouble(v[2]);
  if (eps == -1.0 && PyErr_Occurred()) return NULL;
  a.n_rows = (int32_t)T; a.d = (int32_t)d; a.group = (int32_t)group; a.eps = (float)eps; a.residual_dtype = a.dtype;
  void* p;
  if (rows(&c, x, "x", dtype, T, d, &p, &a.x_stride)) return NULL;
  a.x = p;
  if (vector(&c, weight, "weight", dtype, d, &p)) return NULL;
  a.weight = p;
  if (residual != Py_None) {
    if (layer_type(&c, residual, "residual", &a.residual_dtype, &rdtype) ||
        rows(&c, residual, "residual", rdtype, T, d, &p, &a.residual_stride))
      return NULL;
    a.residual = p;
  }
  if (residual_out != Py_None) {
    if (!rdtype) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "residual_out without residual"); return NULL; }
    if (rows(&c, residual_out, "residual_out", rdtype, T, d, &a.residual_out, &a.residual_out_stride)) return NULL;
  }
  if (out != Py_None && rows(&c, out, "out", dtype, T, d, &a.out, &a.out_stride)) return NULL;
  if ((out8 == Py_None) != (scales == Py_None)) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "out8 and scales go together"); return NULL; }
  if (out8 != Py_None) {
    if (rows(&c, out8, "out8", d_e4m3, T, d, &a.out8, &a.out8_stride) ||
        rows(&c, scales, "scales", d_f32, T, group ? (d + group - 1) / group : 1, &p, &a.scales_stride))
      return NULL;
    a.scales = (float*)p;
  }
  void* st;
  long back;
  int32_t status;
  if (begin(&c, v[9], &st, &back)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = f_rms_norm(&a, st);
  Py_END_ALLOW_THREADS
  return end(&c, back, status);
}

/* route(gate, logits, experts, weights, bias, expert_to_slot, slots, stream) */
static PyObject* py_route(PyObject* self, PyObject* const* v, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "eight arguments expected");
  Call c = {"swapmoe_route", -1};
  PyObject *logits = v[1], *experts = v[2], *weights = v[3], *bias = v[4], *table = v[5], *slots = v[6];
  int dims;
  int64_t size[2], stride[2], ks[2], kstride[2], row_stride;
  void *lp, *ep, *wp, *bp = NULL, *tp = NULL, *sp = NULL, *st;
  long back;
  int32_t status;
  swapmoe_gate_t gate;
  Py_buffer buf;
  if (PyObject_GetBuffer(v[0], &buf, PyBUF_SIMPLE)) return NULL;
  const int fits = buf.len == (Py_ssize_t)sizeof(gate);
  if (fits) gate = *(const swapmoe_gate_t*)buf.buf;
  PyBuffer_Release(&buf);
  if (!fits) return PyErr_Format(PyExc_TypeError, "a Gate expected");
  if (sizes(&c, logits, "logits", &dims, size, stride)) return NULL;
  if (dims != 2) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "logits: [T, E] expected"); return NULL; }
  if (sizes(&c, experts, "experts", &dims, ks, kstride)) return NULL;
  if (dims != 2) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "experts: [T, top_k] expected"); return NULL; }
  const int64_t T = size[0], E = size[1], k = ks[1];
  if (rows(&c, logits, "logits", d_f32, T, E, &lp, &row_stride)) return NULL;
  if ((table == Py_None) != (slots == Py_None)) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "expert_to_slot and slots go together"); return NULL; }
  if (vector(&c, experts, "experts", d_i32, T * k, &ep) || vector(&c, weights, "weights", d_f32, T * k, &wp) ||
      (bias != Py_None && vector(&c, bias, "bias", d_f32, E, &bp)) ||
      (table != Py_None && (vector(&c, table, "expert_to_slot", d_i32, E, &tp) || vector(&c, slots, "slots", d_i32, T * k, &sp))))
    return NULL;
  if (begin(&c, v[7], &st, &back)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = f_route(&gate, lp, row_stride, bp, tp, (int32_t)T, (int32_t)E, (int32_t)k, ep, wp, sp, st);
  Py_END_ALLOW_THREADS
  return end(&c, back, status);
}

/* adapters_forward(handle, device, dtype, d_in, d_out, x, ids, y, out, x_scales, stream) */
static PyObject* py_adapters_forward(PyObject* self, PyObject* const* v, Py_ssize_t n) {
  if (n != 11) return PyErr_Format(PyExc_TypeError, "eleven arguments expected");
  Call c = {"swapmoe_adapters_forward", -1};
  PyObject *dtype = v[2], *x = v[5], *ids = v[6], *y = v[7], *out = v[8], *x_scales = v[9];
  int dims;
  int64_t device, d_in, d_out, size[2], stride[2], xs, ys = 0, os;
  void *xp, *ip, *yp = NULL, *op, *sp = NULL, *st;
  long back;
  int32_t status;
  if (integer(v[1], &device) || integer(v[3], &d_in) || integer(v[4], &d_out)) return NULL;
  void* bank = v[0] == Py_None ? NULL : PyLong_AsVoidPtr(v[0]);
  if (PyErr_Occurred() || sizes(&c, x, "x", &dims, size, stride)) return NULL;
  if (dims != 2) { refuse(&c, SWAPMOE_ERR_INVALID_ARG, "x: [T, d_in] expected"); return NULL; }
  const int64_t T = size[0];
  c.device = (long)device;
  if (rows(&c, x, "x", x_scales == Py_None ? dtype : d_e4m3, T, d_in, &xp, &xs) || vector(&c, ids, "ids", d_i32, T, &ip) ||
      (x_scales != Py_None && vector(&c, x_scales, "x_scales", d_f32, T, &sp)) ||
      (y != Py_None && rows(&c, y, "y", dtype, T, d_out, &yp, &ys)) || rows(&c, out, "out", dtype, T, d_out, &op, &os))
    return NULL;
  if (begin(&c, v[10], &st, &back)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = f_adapters(bank, xp, xs, sp, ip, yp, ys, op, os, (int32_t)T, st);
  Py_END_ALLOW_THREADS
  return end(&c, back, status);
}

/* init(fail, (addresses of the library's functions), (torch's types), (torch's device and stream functions)) */
static PyObject* py_init(PyObject* self, PyObject* args) {
  PyObject *e, *a[3], *t[4], *d[3];
  if (!PyArg_ParseTuple(args, "O(OOO)(OOOO)(OOO)", &e, &a[0], &a[1], &a[2], &t[0], &t[1], &t[2], &t[3], &d[0], &d[1], &d[2])) return NULL;
  f_rms_norm = (rms_norm_fn)PyLong_AsVoidPtr(a[0]);
  f_route = (route_fn)PyLong_AsVoidPtr(a[1]);
  f_adapters = (adapters_fn)PyLong_AsVoidPtr(a[2]);
  if (PyErr_Occurred()) return NULL;
  fail = Py_NewRef(e);                              /* (kept for the life of the process, like the functions themselves) */
  d_f32 = Py_NewRef(t[0]); d_bf16 = Py_NewRef(t[1]); d_e4m3 = Py_NewRef(t[2]); d_i32 = Py_NewRef(t[3]);
  get_device_fn = Py_NewRef(d[0]); set_device_fn = Py_NewRef(d[1]); raw_stream_fn = Py_NewRef(d[2]);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"init", py_init, METH_VARARGS, NULL},
    {"rms_norm", (PyCFunction)(void (*)(void))py_rms_norm, METH_FASTCALL, NULL},
    {"route", (PyCFunction)(void (*)(void))py_route, METH_FASTCALL, NULL},
    {"adapters_forward", (PyCFunction)(void (*)(void))py_adapters_forward, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_numel = PyUnicode_InternFromString("numel");
  return PyModule_Create(&module);
}
