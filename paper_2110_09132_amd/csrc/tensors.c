/* The binding's marshalling of lists of tensors (adamw_step): checks every
 * tensor and writes the emb_adamw_tensor structs, in one call.  In Python each
 * tensor costs five attribute reads of 50 to 80 ns (73 parameters with their
 * gradients, moments and copies: 100 us a step, more than the GPU needs for
 * small ones); here about 20 ns.
 *
 * The tensors are read through the table of C functions that DLPack defines for
 * such calls (`__dlpack_c_exchange_api__` of the tensor type): addresses and
 * shapes that are valid while the call runs, no references kept.  Held inside
 * the interpreter's lock (ctypes.PyDLL). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/dlpack.h>

#include "emb.h"

/* The function that reads a tensor, of the table in a `dlpack_exchange_api`
 * capsule; NULL where its version is another or it has none. */
void *emb_tensor_reader(PyObject *capsule) {
  const DLPackExchangeAPI *api = (const DLPackExchangeAPI *)PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
  if (api == NULL) {
    PyErr_Clear();
    return NULL;
  }
  return api->header.version.major == DLPACK_MAJOR_VERSION ? (void *)api->dltensor_from_py_object_no_sync : NULL;
}

typedef struct {
  DLPackDLTensorFromPyObjectNoSync read;
  PyObject *type, *subtype; /* the types of tensors that are read here */
  Py_ssize_t n;
} Reader;

/* Number of elements of a contiguous device tensor of this element type, and its address; -1 otherwise. */
static int64_t one(const Reader *r, PyObject *o, int code, int bits, void **data) {
  DLTensor t;
  PyObject *type = (PyObject *)Py_TYPE(o);
  if (type != r->type && type != r->subtype) return -1;
  if (r->read(o, &t) != 0) {
    PyErr_Clear();
    return -1;
  }
  if (t.device.device_type != kDLROCM && t.device.device_type != kDLCUDA) return -1;
  if (t.dtype.code != code || t.dtype.bits != bits || t.dtype.lanes != 1) return -1;
  int64_t n = 1, dense = 1;
  for (int d = t.ndim - 1; d >= 0; --d) {
    if (t.strides != NULL && t.shape[d] != 1 && t.strides[d] != n) dense = 0;
    n *= t.shape[d];
  }
  if (n != 0 && !dense) return -1;
  *data = n == 0 ? NULL : (char *)t.data + t.byte_offset;
  return n;
}

/* Addresses of a list's tensors into the structs' field at byte `at`; sizes are
 * taken from the structs (each tensor must have `per` elements for every started
 * `block` of them), or written to them where per is 0. */
static int column(const Reader *r, PyObject *list, int code, int bits, emb_adamw_tensor *out, size_t at, int64_t per,
                  int64_t block) {
  int ok = 0;
  PyObject *seq = PySequence_Fast(list, "a list of tensors");
  if (seq == NULL) {
    PyErr_Clear();
    return 0;
  }
  if (PySequence_Fast_GET_SIZE(seq) == r->n) {
    PyObject **items = PySequence_Fast_ITEMS(seq);
    ok = 1;
    for (Py_ssize_t k = 0; ok && k < r->n; ++k) {
      void *data = NULL;
      const int64_t n = one(r, items[k], code, bits, &data);
      if (n < 0)
        ok = 0;
      else if (per == 0)
        out[k].n = n;
      else
        ok = n == (out[k].n + block - 1) / block * per;
      *(void **)((char *)&out[k] + at) = data;
    }
  }
  Py_DECREF(seq);
  return ok;
}

/* Fills out[n] from the lists (scales and copies may be None).  Returns the
 * gradients' type (EMB_F32 or EMB_BF16), or -1 where a tensor does not fit the
 * call or cannot be read here: the caller then goes through them itself. */
int emb_adamw_tensors(void *read, PyObject *type, PyObject *subtype, PyObject *params, PyObject *grads,
                      PyObject *exp_avgs, PyObject *exp_avg_sqs, PyObject *scales, PyObject *copies, Py_ssize_t n,
                      emb_adamw_tensor *out) {
  const Reader r = {(DLPackDLTensorFromPyObjectNoSync)read, type, subtype, n};
  const int eight = scales != Py_None;
#define FIELD(f) offsetof(emb_adamw_tensor, f)
  int gt = EMB_F32;
  if (!column(&r, params, kDLFloat, 32, out, FIELD(param), 0, 1)) return -1;
  if (!column(&r, grads, kDLFloat, 32, out, FIELD(grad), 1, 1)) {
    if (!column(&r, grads, kDLBfloat, 16, out, FIELD(grad), 1, 1)) return -1;
    gt = EMB_BF16;
  }
  if (!column(&r, exp_avgs, eight ? kDLFloat8_e4m3fn : kDLFloat, eight ? 8 : 32, out, FIELD(exp_avg), 1, 1) ||
      !column(&r, exp_avg_sqs, eight ? kDLFloat8_e5m2 : kDLFloat, eight ? 8 : 32, out, FIELD(exp_avg_sq), 1, 1))
    return -1;
  if (eight && !column(&r, scales, kDLFloat, 32, out, FIELD(scales), 2, EMB_ADAMW_BLOCK)) return -1;
  if (copies != Py_None && !column(&r, copies, kDLBfloat, 16, out, FIELD(copy), 1, 1)) return -1;
#undef FIELD
  return gt;
}
