/* The short way from the dense operators' binding (dense.py) to the C ABI: reads
 * the tensors, checks them and makes the call, without a step in Python between.
 * A call of few rows or of many small tensors is bound by the host, and there
 * every attribute read costs 50 to 80 ns and a ctypes call more than 1 us: a
 * layer norm with its six tensors 7.1 us per call through Python and ctypes, of
 * which the launch is 3; an AdamW step of 25 tensors 33 us.
 *
 * Every function returns the call's status, or -1 where an argument is not what
 * the call takes or cannot be read here: the binding then goes the long way,
 * which accepts the same and says what is wrong.
 *
 * Tensors are read through the table of C functions that DLPack defines for such
 * calls (`__dlpack_c_exchange_api__` of the tensor type): addresses and shapes
 * that are valid while the caller holds the tensors; nothing is kept. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/dlpack.h>
#include <stddef.h>
#include <stdlib.h>

#include "emb.h"

static DLPackDLTensorFromPyObjectNoSync reader; /* NULL: no tensor is read here */
static PyObject *tensor_type, *parameter_type;  /* the types that are */

enum { OTHER = -1, I32 = 100, E4M3, E5M2, BYTES }; /* element types beside EMB_F32 and EMB_BF16 */

static int element(DLDataType t) {
  if (t.lanes != 1) return OTHER;
  if (t.code == kDLFloat && t.bits == 32) return EMB_F32;
  if (t.code == kDLBfloat && t.bits == 16) return EMB_BF16;
  if (t.code == kDLInt && t.bits == 32) return I32;
  if (t.code == kDLUInt && t.bits == 8) return BYTES;
  if (t.code == kDLFloat8_e4m3fn && t.bits == 8) return E4M3;
  if (t.code == kDLFloat8_e5m2 && t.bits == 8) return E5M2;
  return OTHER;
}

/* A device tensor; returns its element type, or OTHER where it is none. */
static int take(PyObject *o, DLTensor *t) {
  PyObject *type = (PyObject *)Py_TYPE(o);
  if (type != tensor_type && type != parameter_type) return OTHER;
  if (reader(o, t) != 0) {
    PyErr_Clear();
    return OTHER;
  }
  if (t->device.device_type != kDLROCM && t->device.device_type != kDLCUDA) return OTHER;
  return element(t->dtype);
}
static void *address(const DLTensor *t) { return t->data == NULL ? NULL : (char *)t->data + t->byte_offset; }

/* Elements of a contiguous tensor; -1 where it is not contiguous. */
static int64_t elements(const DLTensor *t) {
  int64_t n = 1;
  int dense = 1;
  for (int d = t->ndim - 1; d >= 0; --d) {
    if (t->strides != NULL && t->shape[d] != 1 && t->strides[d] != n) dense = 0;
    n *= t->shape[d];
  }
  return n == 0 || dense ? n : -1;
}
static int64_t stride(const DLTensor *t, int d) {
  if (t->strides != NULL) return t->strides[d];
  int64_t s = 1;
  for (int i = t->ndim - 1; i > d; --i) s *= t->shape[i];
  return s;
}

/* A contiguous buffer of at least `least` elements of one type; None is NULL where it may be. */
static int buffer(PyObject *o, int type, int64_t least, int optional, void **p) {
  DLTensor t;
  if (o == Py_None) {
    *p = NULL;
    return optional;
  }
  if (take(o, &t) != type || elements(&t) < least) return 0;
  *p = address(&t);
  return 1;
}

/* Rows of fp32 or bf16 that may lie apart. */
typedef struct {
  void *p;
  int type;
  int64_t n, D, ld;
} Rows;
static int rows(PyObject *o, Rows *r) {
  DLTensor t;
  r->type = take(o, &t);
  if ((r->type != EMB_F32 && r->type != EMB_BF16) || t.ndim != 2) return 0;
  r->n = t.shape[0];
  r->D = t.shape[1];
  if (r->D > 1 && stride(&t, 1) != 1) return 0;
  r->ld = r->n > 1 ? stride(&t, 0) : r->D;
  r->p = address(&t);
  return r->n < (1 << 30) && r->D < (1 << 30);
}

static int number(PyObject *o, int64_t *x) {
  *x = PyLong_AsLongLong(o);
  return !(*x == -1 && PyErr_Occurred());
}
static int real(PyObject *o, double *x) {
  *x = PyFloat_AsDouble(o);
  return !(*x == -1.0 && PyErr_Occurred());
}

static PyObject *no(void) {
  PyErr_Clear();
  return PyLong_FromLong(-1);
}
/* The interpreter's lock is given up while the call is enqueued. */
#define CALL(expression)                    \
  do {                                      \
    int status_;                            \
    Py_BEGIN_ALLOW_THREADS                  \
    status_ = (expression);                 \
    Py_END_ALLOW_THREADS                    \
    return PyLong_FromLong(status_);        \
  } while (0)
#define ARGUMENTS(count) \
  if (reader == NULL || n_args != (count)) return no()

/* use(capsule, Tensor, Parameter): reads tensors from now on through the capsule's functions (None: not here).
 * Returns whether they can be read. */
static PyObject *use(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
  (void)self;
  if (n_args != 3) return no();
  reader = NULL;
  if (a[0] != Py_None) {
    const DLPackExchangeAPI *api = (const DLPackExchangeAPI *)PyCapsule_GetPointer(a[0], "dlpack_exchange_api");
    if (api == NULL)
      PyErr_Clear();
    else if (api->header.version.major == DLPACK_MAJOR_VERSION)
      reader = api->dltensor_from_py_object_no_sync;
  }
  Py_INCREF(a[1]);
  Py_INCREF(a[2]);
  Py_XSETREF(tensor_type, a[1]);
  Py_XSETREF(parameter_type, a[2]);
  return PyBool_FromLong(reader != NULL);
}

/* The rows of x, or the ids' rows of the table x: T, and V (0 without ids). */
static int source(PyObject *x, PyObject *ids, Rows *r, void **id, int64_t *T, int64_t *V) {
  DLTensor t;
  if (!rows(x, r)) return 0;
  *id = NULL;
  *T = r->n;
  *V = 0;
  if (ids == Py_None) return 1;
  if (take(ids, &t) != I32 || (*T = elements(&t)) < 0 || *T >= (1 << 30)) return 0;
  *id = address(&t);
  *V = r->n;
  return *T == 0 || *id != NULL;
}

/* layer_norm(x, weight, bias, eps, ids, y, mean, rstd, dev_status, stream) */
static PyObject *layer_norm(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
  (void)self;
  ARGUMENTS(10);
  Rows x, y;
  void *w, *b, *ids, *mean, *rstd, *status;
  int64_t T, V, stream;
  double eps;
  if (!source(a[0], a[4], &x, &ids, &T, &V) || !buffer(a[1], EMB_F32, x.D, 1, &w) ||
      !buffer(a[2], EMB_F32, x.D, 1, &b) || !real(a[3], &eps) || !rows(a[5], &y) || y.n != T || y.D != x.D ||
      y.ld < y.D || !buffer(a[6], EMB_F32, T, 0, &mean) || !buffer(a[7], EMB_F32, T, 0, &rstd) ||
      !buffer(a[8], I32, 1, 1, &status) || !number(a[9], &stream))
    return no();
  CALL(emb_layer_norm(x.p, x.type, x.ld, ids, V, (int32_t)T, (int32_t)x.D, w, b, eps, y.p, y.type, y.ld, mean, rstd,
                      status, (void *)stream));
}

/* layer_norm_backward(dy, x, mean, rstd, weight, ids, dx, dweight, dbias, workspace, dev_status, stream) */
static PyObject *layer_norm_backward(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
  (void)self;
  ARGUMENTS(12);
  Rows dy, x, dx = {NULL, 0, 0, 0, 0};
  void *mean, *rstd, *w, *ids, *dw, *db, *ws, *status;
  int64_t T, V, stream;
  DLTensor t;
  if (!rows(a[0], &dy) || !source(a[1], a[5], &x, &ids, &T, &V) || dy.n != T || dy.D != x.D ||
      !buffer(a[2], EMB_F32, T, 0, &mean) || !buffer(a[3], EMB_F32, T, 0, &rstd) ||
      !buffer(a[4], EMB_F32, x.D, 1, &w) || !buffer(a[7], EMB_F32, x.D, 1, &dw) ||
      !buffer(a[8], EMB_F32, x.D, 1, &db) || !buffer(a[10], I32, 1, 1, &status) || !number(a[11], &stream))
    return no();
  dx.ld = x.D;
  if (a[6] != Py_None &&
      (!rows(a[6], &dx) || dx.n != T || dx.D != x.D || dx.type != dy.type || dx.ld < dx.D))
    return no();
  if (a[9] == Py_None || take(a[9], &t) != BYTES || elements(&t) < 0) return no();
  ws = address(&t);
  CALL(emb_layer_norm_backward(dy.p, dy.type, dy.ld, x.p, x.type, x.ld, ids, V, (int32_t)T, (int32_t)x.D, w, mean,
                               rstd, dx.p, dx.ld, dw, db, ws, (size_t)elements(&t), status, (void *)stream));
}

/* relative_bias(table, bucket_of, Q, K, q0, out, dev_status, stream) */
static PyObject *relative_bias(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
  (void)self;
  ARGUMENTS(8);
  DLTensor table, map, out;
  void *status;
  int64_t Q, K, q0, stream;
  if (take(a[0], &table) != EMB_F32 || table.ndim != 2 || elements(&table) < 0 || take(a[1], &map) != I32 ||
      !number(a[2], &Q) || !number(a[3], &K) || !number(a[4], &q0) || !buffer(a[6], I32, 1, 1, &status) ||
      !number(a[7], &stream))
    return no();
  const int64_t places = elements(&map), B = table.shape[0], H = table.shape[1];
  const int type = take(a[5], &out);
  if (places % 2 != 1 || places >= INT32_MAX || (type != EMB_F32 && type != EMB_BF16) || out.ndim != 3 ||
      out.shape[0] != H || out.shape[1] != Q || out.shape[2] != K || (K > 1 && stride(&out, 2) != 1) ||
      B >= INT32_MAX || H >= INT32_MAX || Q >= (1 << 30) || K >= (1 << 30))
    return no();
  CALL(emb_relative_bias(address(&table), (int32_t)B, (int32_t)H, address(&map), (int32_t)(places / 2), (int32_t)Q,
                         (int32_t)K, q0, address(&out), type, Q > 1 ? stride(&out, 1) : K, stride(&out, 0), status,
                         (void *)stream));
}

/* relative_bias_backward(grad, bucket_of, num_buckets, q0, out, workspace, dev_status, stream) */
static PyObject *relative_bias_backward(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
  (void)self;
  ARGUMENTS(8);
  DLTensor g, map, ws;
  void *out, *status;
  int64_t B, q0, stream;
  const int type = take(a[0], &g);
  if ((type != EMB_F32 && type != EMB_BF16) || (g.ndim != 3 && g.ndim != 4) || take(a[1], &map) != I32 ||
      !number(a[2], &B) || !number(a[3], &q0) || B < 1 || B >= INT32_MAX || take(a[5], &ws) != BYTES ||
      elements(&ws) < 0 || !buffer(a[6], I32, 1, 1, &status) || !number(a[7], &stream))
    return no();
  const int h = g.ndim - 3;  /* the heads' dimension */
  const int64_t places = elements(&map), N = h ? g.shape[0] : 1, H = g.shape[h], Q = g.shape[h + 1],
                K = g.shape[h + 2];
  if (places % 2 != 1 || places >= INT32_MAX || (K > 1 && stride(&g, h + 2) != 1) || N >= INT32_MAX ||
      H >= INT32_MAX || Q >= (1 << 30) || K >= (1 << 30) || !buffer(a[4], EMB_F32, B * H, 0, &out))
    return no();
  CALL(emb_relative_bias_backward(address(&g), type, (int32_t)N, (int32_t)H, (int32_t)Q, (int32_t)K,
                                  h ? stride(&g, 0) : 0, stride(&g, h), stride(&g, h + 1), address(&map),
                                  (int32_t)(places / 2), (int32_t)B, q0, out, address(&ws), (size_t)elements(&ws),
                                  status, (void *)stream));
}

/* Addresses of a list's n tensors into one field of the structs.  per == 0: the
 * field is param, and the sizes are written; else each tensor has `per` elements
 * for every started `block` of its parameter's. */
static int column(PyObject *list, Py_ssize_t n, int type, emb_adamw_tensor *out, size_t field, int64_t per,
                  int64_t block) {
  int ok = 0;
  PyObject *seq = PySequence_Fast(list, "a list of tensors");
  if (seq == NULL) {
    PyErr_Clear();
    return 0;
  }
  if (PySequence_Fast_GET_SIZE(seq) == n) {
    PyObject **items = PySequence_Fast_ITEMS(seq);
    ok = 1;
    for (Py_ssize_t k = 0; ok && k < n; ++k) {
      DLTensor t;
      const int64_t size = take(items[k], &t) == type ? elements(&t) : -1;
      if (size < 0) {
        ok = 0;
        break;
      }
      if (per == 0)
        out[k].n = size;
      else
        ok = size == (out[k].n + block - 1) / block * per;
      *(void **)((char *)&out[k] + field) = address(&t);
    }
  }
  Py_DECREF(seq);
  return ok;
}

/* adamw_step(params, grads, exp_avgs, exp_avg_sqs, scales, copies, lr, beta1, beta2, eps, weight_decay, step, seed,
 *            coeffs, grad_scale, dev_status, stream) */
static PyObject *adamw_step(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
  (void)self;
  ARGUMENTS(17);
  const Py_ssize_t n = PyObject_Size(a[0]);
  double h[5];
  int64_t step, stream;
  void *coeffs, *scale, *status;
  if (n < 0 || n >= INT32_MAX) return no();
  for (int k = 0; k < 5; ++k)
    if (!real(a[6 + k], &h[k])) return no();
  const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[12]);
  if (PyErr_Occurred() || !number(a[11], &step) || !buffer(a[13], EMB_F32, EMB_ADAMW_COEFFS_WORDS, 1, &coeffs) ||
      !buffer(a[14], EMB_F32, 1, 1, &scale) || !buffer(a[15], I32, 1, 1, &status) || !number(a[16], &stream))
    return no();
  emb_adamw_tensor few[64], *t = few;
  if (n > 64 && (t = (emb_adamw_tensor *)malloc((size_t)n * sizeof(*t))) == NULL) return no();
  for (Py_ssize_t k = 0; k < n; ++k) t[k] = (emb_adamw_tensor){0};
  const int eight = a[4] != Py_None;
  int type = EMB_F32;
#define FIELD(f) offsetof(emb_adamw_tensor, f)
  int ok = column(a[0], n, EMB_F32, t, FIELD(param), 0, 1);
  if (ok && !column(a[1], n, EMB_F32, t, FIELD(grad), 1, 1)) {
    type = EMB_BF16;
    ok = column(a[1], n, EMB_BF16, t, FIELD(grad), 1, 1);
  }
  ok = ok && column(a[2], n, eight ? E4M3 : EMB_F32, t, FIELD(exp_avg), 1, 1) &&
       column(a[3], n, eight ? E5M2 : EMB_F32, t, FIELD(exp_avg_sq), 1, 1) &&
       (!eight || column(a[4], n, EMB_F32, t, FIELD(scales), 2, EMB_ADAMW_BLOCK)) &&
       (a[5] == Py_None || column(a[5], n, EMB_BF16, t, FIELD(copy), 1, 1));
#undef FIELD
  int status_code = -1;
  if (ok) {
    Py_BEGIN_ALLOW_THREADS
    status_code = emb_adamw_step(t, (int32_t)n, type, eight ? 8 : 32, h[0], h[1], h[2], h[3], h[4], step, seed,
                                 coeffs, scale, status, (void *)stream);
    Py_END_ALLOW_THREADS
  }
  if (t != few) free(t);
  PyErr_Clear();
  return PyLong_FromLong(status_code);
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(use),           METHOD(layer_norm),
                                METHOD(layer_norm_backward), METHOD(relative_bias),
                                METHOD(relative_bias_backward), METHOD(adamw_step),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
