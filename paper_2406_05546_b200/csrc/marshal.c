/* Argument marshalling of the calls a training loop makes every tick, as a CPython extension: snapshots in and out of their
 * ctypes structures, numpy arrays by the buffer protocol, the results as Python objects.  Through ctypes alone these calls
 * cost the host more than the library's own work (measured per call, ctypes -> here: pull 0.9 -> 0.3 us, reserve 3.6 -> 0.9,
 * enqueue 9 -> 2, apply 5 -> 1.5, the grad step's arguments 20 -> 8).  Arrays that already have their type and layout are read
 * where they lie, and a list of versions is read element by element: only the rest goes through numpy.  No step of the method
 * happens here. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "ps.h"

static int32_t (*f_pull)(ps_ctx*, int32_t, int32_t, ps_snapshot*);
static int32_t (*f_reserve)(ps_ctx*, int32_t, int64_t*);
static int32_t (*f_grad)(ps_ctx*, int32_t, int32_t, const ps_snapshot*, const int32_t*, const float*, const int32_t*, uint64_t,
                         uint64_t, const int64_t*, float*, float*, int32_t*);
static int32_t (*f_summed)(ps_ctx*, int32_t, int32_t, const ps_snapshot*, const int32_t*, const float*, const int32_t*, uint64_t,
                           uint64_t, float*, float*, int32_t*);
static int32_t (*f_eval)(ps_ctx*, int32_t, int32_t, const ps_snapshot*, const float*, const int32_t*, float*, int32_t*, int32_t*);
static int32_t (*f_enqueue)(ps_ctx*, int32_t, const int64_t*, const float*, const int32_t*, const uint64_t*, uint64_t);
static int32_t (*f_apply)(ps_ctx*, ps_mode, float, float, const int32_t*, ps_apply_result*);
static int32_t (*f_apply_stale)(ps_ctx*, ps_mode, float, float, const int32_t*, float, float, ps_apply_result*);
static int32_t (*f_apply_summed)(ps_ctx*, const float*, int32_t, float, float, ps_apply_result*);
static int32_t (*f_apply_adamw)(ps_ctx*, ps_mode, const ps_adamw_hyper*, double, float*, float*, float, const int32_t*, float, ps_apply_result*);
static int32_t (*f_adamw_step)(ps_adamw*, const ps_adamw_hyper*);
static int32_t (*f_dense_forward)(const ps_dense_layer*, const ps_dense_output*);
static int32_t (*f_dense_workspace)(const ps_dense_layer*, const void*, int64_t, uint64_t*);
static int32_t (*f_dense_backward)(const ps_dense_layer*, const ps_dense_gradients*);
static const char* (*f_error)(ps_ctx*);
static PyObject *snapshot_type, *error_type;
static PyObject *as_array;       /* as_array(object, kind): numpy's conversion to a contiguous array */
static PyObject *as_snapshots;   /* as_snapshots(sequence, n): ctypes' conversion to an array of n structures */
static PyObject *k_applied, *k_version, *k_checkpointed, *k_replicated;

static PyObject* raise(int32_t rc) {
  PyObject* e = PyObject_CallFunction(error_type, "is", (int)rc, f_error(NULL));
  if (e) { PyErr_SetObject(error_type, e); Py_DECREF(e); }
  return NULL;
}

/* Integer arguments: anything int() takes, wrapped like a C conversion, as ctypes does it. */
static int as_u64(PyObject* o, uint64_t* v) {
  PyObject* i = PyNumber_Long(o);
  if (!i) return -1;
  *v = PyLong_AsUnsignedLongLongMask(i);
  Py_DECREF(i);
  return PyErr_Occurred() ? -1 : 0;
}
static int i32(PyObject* o, int32_t* v) {
  uint64_t w;
  if (as_u64(o, &w)) return -1;
  *v = (int32_t)(uint32_t)w;
  return 0;
}
static int as_ptr(PyObject* o, void** p) {         /* None or an address */
  if (o == Py_None) { *p = NULL; return 0; }
  *p = PyLong_AsVoidPtr(o);
  return !*p && PyErr_Occurred() ? -1 : 0;
}
static int as_float(PyObject* o, float* v) {       /* anything float() takes */
  PyObject* f = PyNumber_Float(o);
  if (!f) return -1;
  *v = (float)PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  return 0;
}

static int as_double(PyObject* o, double* v) {
  PyObject* f = PyNumber_Float(o);
  if (!f) return -1;
  *v = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  return 0;
}
/* (lr, beta1, beta2, eps, step, clip_norm, grad_scale) from a[0] on */
static int hyper(PyObject* const* a, ps_adamw_hyper* h) {
  uint64_t step;
  memset(h, 0, sizeof(*h));
  if (as_double(a[0], &h->lr) || as_double(a[1], &h->beta1) || as_double(a[2], &h->beta2) || as_double(a[3], &h->eps) || as_u64(a[4], &step) ||
      as_double(a[5], &h->clip_norm) || as_double(a[6], &h->grad_scale))
    return -1;
  h->step = (int64_t)step;
  return 0;
}

/* The types of the library's integer arrays. */
enum { I32, I64, U64 };

/* A contiguous one-dimensional array of the given type, or None.  The buffer keeps whatever holds the items alive. */
static int array(PyObject* o, Py_buffer* b, int kind) {
  b->obj = NULL;
  b->buf = NULL;
  b->len = 0;
  if (o == Py_None) return 0;
  if (PyObject_CheckBuffer(o)) {
    if (PyObject_GetBuffer(o, b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) == 0) {
      const char f = b->ndim == 1 && b->format && b->format[0] && !b->format[1] ? b->format[0] : 0;
      if (b->itemsize == (kind == I32 ? 4 : 8) && (kind == U64 ? f == 'L' || f == 'Q' : f == 'i' || f == 'l' || f == 'q')) return 0;
      PyBuffer_Release(b);
    } else PyErr_Clear();
  }
  PyObject* c = PyObject_CallFunction(as_array, "Oi", o, kind);
  if (!c) { b->obj = NULL; return -1; }
  const int rc = PyObject_GetBuffer(c, b, PyBUF_C_CONTIGUOUS);
  Py_DECREF(c);
  return rc;
}
static void done(Py_buffer* b) { if (b->obj) PyBuffer_Release(b); }

static int long_enough(const Py_buffer* b, Py_ssize_t n, Py_ssize_t item) {
  if (!b->obj || b->len >= n * item) return 1;
  PyErr_SetString(PyExc_ValueError, "array is too short");
  return 0;
}

/* The snapshots of a call, out of their structures.  Anything but a list or tuple of n Snapshots goes through ctypes, which
 * converts or refuses it. */
static int snapshots(PyObject* seq, Py_ssize_t n, ps_snapshot* out) {
  Py_buffer b;
  Py_ssize_t i = 0;
  if ((PyList_CheckExact(seq) || PyTuple_CheckExact(seq)) && PySequence_Fast_GET_SIZE(seq) == n) {
    for (; i < n; ++i) {
      PyObject* o = PySequence_Fast_GET_ITEM(seq, i);
      if ((PyObject*)Py_TYPE(o) != snapshot_type) break;
      if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) return -1;
      out[i] = *(const ps_snapshot*)b.buf;
      PyBuffer_Release(&b);
    }
    if (i == n) return 0;
  }
  PyObject* c = PyObject_CallFunction(as_snapshots, "On", seq, n);
  if (!c) return -1;
  const int rc = PyObject_GetBuffer(c, &b, PyBUF_SIMPLE);
  Py_DECREF(c);
  if (rc) return -1;
  memcpy(out, b.buf, (size_t)n * sizeof(ps_snapshot));
  PyBuffer_Release(&b);
  return 0;
}

static PyObject* result(const ps_apply_result* r) {
  PyObject* d = PyDict_New();
  PyObject* v[4] = {PyLong_FromLongLong(r->applied), PyLong_FromUnsignedLongLong(r->new_version), PyLong_FromLong(r->checkpointed), PyLong_FromLong(r->replicated)};
  PyObject* k[4] = {k_applied, k_version, k_checkpointed, k_replicated};
  int bad = !d;
  for (int i = 0; i < 4; ++i) {
    if (!v[i] || bad || PyDict_SetItem(d, k[i], v[i])) bad = 1;
    Py_XDECREF(v[i]);
  }
  if (bad) { Py_XDECREF(d); return NULL; }
  return d;
}

/* The other threads run while the library works (it may wait for room in a stream). */
#define CALL(expr) Py_BEGIN_ALLOW_THREADS rc = (expr); Py_END_ALLOW_THREADS
#define WANT(n) if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return NULL; }

static PyObject* bind(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(5)
  static const struct { const char* name; void** f; } table[] = {
      {"ps_pull_snapshot", (void**)&f_pull}, {"ps_queue_reserve", (void**)&f_reserve}, {"workers_grad_step", (void**)&f_grad},
      {"workers_grad_step_summed", (void**)&f_summed}, {"workers_eval", (void**)&f_eval}, {"ps_enqueue", (void**)&f_enqueue},
      {"ps_apply", (void**)&f_apply}, {"ps_apply_stale", (void**)&f_apply_stale}, {"ps_apply_summed", (void**)&f_apply_summed}, {"ps_last_error", (void**)&f_error},
      {"ps_apply_adamw", (void**)&f_apply_adamw}, {"ps_adamw_step", (void**)&f_adamw_step},
      {"workers_dense_forward", (void**)&f_dense_forward}, {"workers_dense_backward", (void**)&f_dense_backward},
      {"workers_dense_workspace", (void**)&f_dense_workspace}};
  for (size_t i = 0; i < sizeof(table) / sizeof(table[0]); ++i) {
    PyObject* addr = PyDict_GetItemString(a[0], table[i].name);
    if (!addr) { PyErr_SetString(PyExc_KeyError, table[i].name); return NULL; }
    *table[i].f = PyLong_AsVoidPtr(addr);
    if (!*table[i].f) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, table[i].name); return NULL; }
  }
  Py_INCREF(a[1]);
  Py_XSETREF(snapshot_type, a[1]);
  Py_INCREF(a[2]);
  Py_XSETREF(error_type, a[2]);
  Py_INCREF(a[3]);
  Py_XSETREF(as_array, a[3]);
  Py_INCREF(a[4]);
  Py_XSETREF(as_snapshots, a[4]);
  Py_RETURN_NONE;
}

/* (ctx, worker, lag) -> Snapshot */
static PyObject* pull(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(3)
  void* ctx;
  int32_t worker, lag;
  if (as_ptr(a[0], &ctx) || i32(a[1], &worker) || i32(a[2], &lag)) return NULL;
  PyObject* s = PyObject_CallNoArgs(snapshot_type);
  if (!s) return NULL;
  Py_buffer b;
  if (PyObject_GetBuffer(s, &b, PyBUF_WRITABLE)) { Py_DECREF(s); return NULL; }
  const int32_t rc = f_pull((ps_ctx*)ctx, worker, lag, (ps_snapshot*)b.buf);
  PyBuffer_Release(&b);
  if (rc) { Py_DECREF(s); return raise(rc); }
  return s;
}

/* (ctx, n, ids int64[n]) */
static PyObject* reserve(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(3)
  void* ctx;
  int32_t n;
  Py_buffer b;
  if (as_ptr(a[0], &ctx) || i32(a[1], &n) || PyObject_GetBuffer(a[2], &b, PyBUF_WRITABLE)) return NULL;
  const int32_t rc = f_reserve((ps_ctx*)ctx, n, (int64_t*)b.buf);
  PyBuffer_Release(&b);
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* (ctx, W, b, snaps, worker_ids int32[W], x, y, seed, step, slot_ids int64[W] | None, grads | None, loss, argmax) */
static PyObject* grad_step(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(13)
  void *ctx, *x, *y, *grads, *loss, *argmax;
  int32_t W, b;
  uint64_t seed, step;
  ps_snapshot snaps[PS_MAX_WORKERS];
  Py_buffer ids, slots;
  if (as_ptr(a[0], &ctx) || i32(a[1], &W) || i32(a[2], &b) || as_ptr(a[5], &x) || as_ptr(a[6], &y) || as_u64(a[7], &seed) ||
      as_u64(a[8], &step) || as_ptr(a[10], &grads) || as_ptr(a[11], &loss) || as_ptr(a[12], &argmax))
    return NULL;
  if (W <= PS_MAX_WORKERS && snapshots(a[3], W, snaps)) return NULL;      /* of more workers the library reads nothing: it refuses the call */
  if (array(a[4], &ids, I32)) return NULL;
  if (array(a[9], &slots, I64)) { done(&ids); return NULL; }
  if (!ids.obj || ids.ndim != 1 || ids.len != (Py_ssize_t)W * 4) PyErr_SetString(PyExc_AssertionError, "one worker id per worker is wanted");
  else long_enough(&slots, W, 8);
  if (PyErr_Occurred()) { done(&ids); done(&slots); return NULL; }
  int32_t rc;
  CALL(f_grad((ps_ctx*)ctx, W, b, snaps, (const int32_t*)ids.buf, (const float*)x, (const int32_t*)y, seed, step,
                            (const int64_t*)slots.buf, (float*)grads, (float*)loss, (int32_t*)argmax))
  done(&ids);
  done(&slots);
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* (ctx, W, b, snaps, worker_ids, x, y, seed, step, grad_sum, loss, argmax) */
static PyObject* grad_step_summed(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(12)
  void *ctx, *x, *y, *sum, *loss, *argmax;
  int32_t W, b;
  uint64_t seed, step;
  ps_snapshot snaps[PS_MAX_WORKERS];
  Py_buffer ids;
  if (as_ptr(a[0], &ctx) || i32(a[1], &W) || i32(a[2], &b) || as_ptr(a[5], &x) || as_ptr(a[6], &y) || as_u64(a[7], &seed) ||
      as_u64(a[8], &step) || as_ptr(a[9], &sum) || as_ptr(a[10], &loss) || as_ptr(a[11], &argmax))
    return NULL;
  if (W <= PS_MAX_WORKERS && snapshots(a[3], W, snaps)) return NULL;
  if (array(a[4], &ids, I32)) return NULL;
  if (!long_enough(&ids, W, 4)) { done(&ids); return NULL; }
  int32_t rc;
  CALL(f_summed((ps_ctx*)ctx, W, b, snaps, (const int32_t*)ids.buf, (const float*)x, (const int32_t*)y, seed, step,
                              (float*)sum, (float*)loss, (int32_t*)argmax))
  done(&ids);
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* (ctx, W, b, snaps, x, y, loss, argmax, correct) */
static PyObject* eval(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(9)
  void *ctx, *x, *y, *loss, *argmax, *correct;
  int32_t W, b;
  ps_snapshot snaps[PS_MAX_WORKERS];
  if (as_ptr(a[0], &ctx) || i32(a[1], &W) || i32(a[2], &b) || as_ptr(a[4], &x) || as_ptr(a[5], &y) || as_ptr(a[6], &loss) ||
      as_ptr(a[7], &argmax) || as_ptr(a[8], &correct))
    return NULL;
  if (W <= PS_MAX_WORKERS && snapshots(a[3], W, snaps)) return NULL;
  int32_t rc;
  CALL(f_eval((ps_ctx*)ctx, W, b, snaps, (const float*)x, (const int32_t*)y, (float*)loss, (int32_t*)argmax, (int32_t*)correct))
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* A list of versions, read without an array in between; NULL without an error if it is anything else. */
static uint64_t* version_list(PyObject* o, Py_ssize_t n) {
  if (!PyList_CheckExact(o) || PyList_GET_SIZE(o) < n) return NULL;
  uint64_t* v = PyMem_Malloc((size_t)(n ? n : 1) * sizeof(uint64_t));
  for (Py_ssize_t i = 0; v && i < n; ++i) {
    PyObject* e = PyList_GET_ITEM(o, i);
    v[i] = PyLong_CheckExact(e) ? PyLong_AsUnsignedLongLong(e) : (uint64_t)-1;
    if (v[i] == (uint64_t)-1) { PyErr_Clear(); PyMem_Free(v); return NULL; }
  }
  return v;
}

/* (ctx, slot_ids int64[n] | None, grads | None, worker_ids int32[n], base_versions uint64[n], step) */
static PyObject* enqueue(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(6)
  void *ctx, *grads;
  uint64_t step;
  Py_buffer slots = {0}, ids = {0}, base = {0};
  uint64_t* list = NULL;
  PyObject* ret = NULL;
  if (as_ptr(a[0], &ctx) || as_ptr(a[2], &grads) || as_u64(a[5], &step)) return NULL;
  if (a[3] == Py_None || a[4] == Py_None) { PyErr_SetString(PyExc_TypeError, "worker_ids and base_versions are wanted"); return NULL; }
  if (array(a[3], &ids, I32) || array(a[1], &slots, I64)) goto end;
  const Py_ssize_t n = ids.shape[0];
  if (!(list = version_list(a[4], n)) && array(a[4], &base, U64)) goto end;
  if (!long_enough(&slots, n, 8) || !long_enough(&base, n, 8)) goto end;
  int32_t rc;
  CALL(f_enqueue((ps_ctx*)ctx, (int32_t)n, (const int64_t*)slots.buf, (const float*)grads, (const int32_t*)ids.buf,
                 list ? list : (const uint64_t*)base.buf, step))
  ret = rc ? raise(rc) : Py_NewRef(Py_None);
end:
  PyMem_Free(list);
  done(&slots);
  done(&ids);
  done(&base);
  return ret;
}

/* (ctx, mode, lr, scale, order int32[K] | None) -> dict */
static PyObject* apply(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(5)
  void* ctx;
  int32_t mode;
  float lr, scale;
  Py_buffer order;
  ps_apply_result r = {0, 0, 0, 0};
  if (as_ptr(a[0], &ctx) || i32(a[1], &mode) || as_float(a[2], &lr) || as_float(a[3], &scale) || array(a[4], &order, I32)) return NULL;
  int32_t rc;
  CALL(f_apply((ps_ctx*)ctx, (ps_mode)mode, lr, scale, (const int32_t*)order.buf, &r))
  done(&order);
  return rc ? raise(rc) : result(&r);
}

/* (ctx, mode, lr, scale, order int32[K] | None, clip_norm, staleness_alpha) -> dict */
static PyObject* apply_stale(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(7)
  void* ctx;
  int32_t mode;
  float lr, scale, clip, alpha;
  Py_buffer order;
  ps_apply_result r = {0, 0, 0, 0};
  if (as_ptr(a[0], &ctx) || i32(a[1], &mode) || as_float(a[2], &lr) || as_float(a[3], &scale) || as_float(a[5], &clip) ||
      as_float(a[6], &alpha) || array(a[4], &order, I32))
    return NULL;
  int32_t rc;
  CALL(f_apply_stale((ps_ctx*)ctx, (ps_mode)mode, lr, scale, (const int32_t*)order.buf, clip, alpha, &r))
  done(&order);
  return rc ? raise(rc) : result(&r);
}

/* (ctx, grad_sum, n_workers, lr, scale) -> dict */
static PyObject* apply_summed(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(5)
  void *ctx, *sum;
  int32_t n;
  float lr, scale;
  ps_apply_result r = {0, 0, 0, 0};
  if (as_ptr(a[0], &ctx) || as_ptr(a[1], &sum) || i32(a[2], &n) || as_float(a[3], &lr) || as_float(a[4], &scale)) return NULL;
  int32_t rc;
  CALL(f_apply_summed((ps_ctx*)ctx, (const float*)sum, n, lr, scale, &r))
  return rc ? raise(rc) : result(&r);
}

/* (ctx, mode, lr, beta1, beta2, eps, step, clip_norm, grad_scale, weight_decay, m, v, scale, order int32[K] | None, staleness_alpha) -> dict */
static PyObject* apply_adamw(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(15)
  void *ctx, *pm, *pv;
  int32_t mode;
  ps_adamw_hyper h;
  double decay;
  float scale, alpha;
  Py_buffer order;
  ps_apply_result r = {0, 0, 0, 0};
  if (as_ptr(a[0], &ctx) || i32(a[1], &mode) || hyper(a + 2, &h) || as_double(a[9], &decay) || as_ptr(a[10], &pm) || as_ptr(a[11], &pv) ||
      as_float(a[12], &scale) || as_float(a[14], &alpha) || array(a[13], &order, I32))
    return NULL;
  int32_t rc;
  CALL(f_apply_adamw((ps_ctx*)ctx, (ps_mode)mode, &h, decay, (float*)pm, (float*)pv, scale, (const int32_t*)order.buf, alpha, &r))
  done(&order);
  return rc ? raise(rc) : result(&r);
}

/* (optimizer, lr, beta1, beta2, eps, step, clip_norm, grad_scale, seed, lr_dev | None, skip_nonfinite) */
static PyObject* adamw_step(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(11)
  void *opt, *lr_dev;
  ps_adamw_hyper h;
  if (as_ptr(a[0], &opt) || hyper(a + 1, &h) || as_u64(a[8], &h.seed) || as_ptr(a[9], &lr_dev) || i32(a[10], &h.skip_nonfinite)) return NULL;
  h.lr_dev = (const float*)lr_dev;
  int32_t rc;
  CALL(f_adamw_step((ps_adamw*)opt, &h))
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* A list or tuple of integers, or anything else that holds int32, one per group. */
static int group_ints(PyObject* o, int32_t* out, Py_ssize_t* n) {
  if (PyList_CheckExact(o) || PyTuple_CheckExact(o)) {
    const Py_ssize_t len = PySequence_Fast_GET_SIZE(o);
    Py_ssize_t i = 0;
    for (; i < len && i < PS_MAX_WORKERS; ++i) {
      const long v = PyLong_AsLong(PySequence_Fast_GET_ITEM(o, i));
      if (v == -1 && PyErr_Occurred()) return -1;
      if (v != (int32_t)v) { PyErr_SetString(PyExc_OverflowError, "an int32 is wanted"); return -1; }
      out[i] = (int32_t)v;
    }
    *n = len;
    return 0;
  }
  Py_buffer b;
  if (array(o, &b, I32)) return -1;
  *n = b.len / 4;
  memcpy(out, b.buf, (size_t)(*n < PS_MAX_WORKERS ? *n : PS_MAX_WORKERS) * 4);
  done(&b);
  return 0;
}

/* ---- torch tensors, by their Python attributes (a call's tensors cost 0.5 us each here, 1.1 in Python) ---- */
typedef struct {
  char* p;
  Py_ssize_t dims, size[3];
  int64_t stride[3];
  PyObject* dtype;                /* borrowed: dtypes are singletons that live as long as torch */
} View;

static PyObject *n_shape, *n_stride, *n_data_ptr, *n_dtype, *n_get_device, *t_float32;
static PyObject* allocate;        /* allocate(bytes, device) -> a tensor */

static int view(PyObject* t, const char* name, View* v) {
  PyObject *shape = NULL, *stride = NULL, *ptr = NULL;
  int rc = -1;
  if (!(shape = PyObject_GetAttr(t, n_shape)) || !(stride = PyObject_CallMethodNoArgs(t, n_stride)) || !(ptr = PyObject_CallMethodNoArgs(t, n_data_ptr)) ||
      !(v->dtype = PyObject_GetAttr(t, n_dtype)))
    goto end;
  Py_DECREF(v->dtype);
  if (!PyTuple_Check(shape) || !PyTuple_Check(stride) || (v->dims = PyTuple_GET_SIZE(shape)) < 1 || v->dims > 3 || PyTuple_GET_SIZE(stride) != v->dims) {
    PyErr_Format(PyExc_ValueError, "%s: a tensor of one to three dimensions is wanted", name);
    goto end;
  }
  for (Py_ssize_t i = 0; i < v->dims; ++i) {
    v->size[i] = PyLong_AsSsize_t(PyTuple_GET_ITEM(shape, i));
    v->stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i));
  }
  v->p = (char*)PyLong_AsVoidPtr(ptr);
  rc = PyErr_Occurred() ? -1 : 0;
end:
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  Py_XDECREF(ptr);
  return rc;
}
static int on_device(PyObject* t, const char* name, long device) {
  PyObject* d = PyObject_CallMethodNoArgs(t, n_get_device);
  if (!d) return -1;
  const long is = PyLong_AsLong(d);
  Py_DECREF(d);
  if (is == device && !PyErr_Occurred()) return 0;
  if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: a tensor on cuda device %ld is wanted", name, device);
  return -1;
}

/* A matrix of at least `rows` rows with its columns next to each other; of None: nothing.  Another dtype is refused unless `or_float32`. */
static int rows_of(PyObject* t, const char* name, int64_t rows, int64_t cols, PyObject* dtype, int or_float32, long device, void** p, int64_t* pitch, PyObject** got) {
  *p = NULL;
  *pitch = 0;
  if (t == Py_None) return 0;
  View v;
  if (view(t, name, &v) || on_device(t, name, device)) return -1;
  if (v.dims != 2 || v.size[0] < rows || v.size[1] != cols || (v.stride[1] != 1 && cols > 1) || (v.dtype != dtype && !(or_float32 && v.dtype == t_float32))) {
    PyErr_Format(PyExc_ValueError, "%s: at least [%lld, %lld] of %R, columns next to each other, is wanted", name, (long long)rows, (long long)cols, dtype);
    return -1;
  }
  *p = v.p;
  *pitch = v.size[0] <= 1 && v.stride[0] < cols ? cols : v.stride[0];
  if (got) *got = v.dtype;
  return 0;
}
/* A stack of `count` matrices [d1][d2], or of vectors [d2] (d1 < 0); a single one may lack its first dimension. */
static int stack_of(PyObject* t, const char* name, int64_t count, int64_t d1, int64_t d2, PyObject* dtype, int or_float32, long device, void** p, int64_t* pitch, int64_t* stride,
                    PyObject** got) {
  *p = NULL;
  *pitch = *stride = 0;
  if (t == Py_None) return 0;
  View v;
  if (view(t, name, &v) || on_device(t, name, device)) return -1;
  const Py_ssize_t inner = d1 < 0 ? 1 : 2;
  const int single = count == 1 && v.dims == inner;
  const Py_ssize_t o = single ? 0 : 1;
  if (v.dims != inner + o || (!single && v.size[0] != count) || (d1 >= 0 && v.size[o] != d1) || v.size[v.dims - 1] != d2 || (v.stride[v.dims - 1] != 1 && d2 > 1) ||
      (v.dtype != dtype && !(or_float32 && v.dtype == t_float32))) {
    if (d1 < 0) PyErr_Format(PyExc_ValueError, "%s: [%lld, %lld] of %R, columns next to each other, is wanted", name, (long long)count, (long long)d2, dtype);
    else PyErr_Format(PyExc_ValueError, "%s: [%lld, %lld, %lld] of %R, columns next to each other, is wanted", name, (long long)count, (long long)d1, (long long)d2, dtype);
    return -1;
  }
  *p = v.p;
  *stride = single ? 0 : v.stride[0];
  if (d1 >= 0) *pitch = d1 <= 1 && v.stride[o] < d2 ? d2 : v.stride[o];
  if (got) *got = v.dtype;
  return 0;
}

/* A layer's arguments: a[0] x, a[1] weight, a[2] rows, a[3] weight_of | None, a[4] activation, a[5] the operands' type, a[6] device, a[7] stream. */
#define LAYER_ARGS 8
typedef struct {
  ps_dense_layer l;
  int32_t rows[PS_MAX_WORKERS], weights[PS_MAX_WORKERS];
  int64_t total, groups;
  long device;
  PyObject *dtype, *space;        /* space: the workspace's tensor, or NULL */
} Layer;

static int layer(PyObject* const* a, Layer* y) {
  ps_dense_layer* l = &y->l;
  Py_ssize_t n, nw;
  void *st, *p;
  View w;
  memset(l, 0, sizeof(*l));
  y->space = NULL;
  y->device = PyLong_AsLong(a[6]);
  if (a[2] == Py_None) PyErr_SetString(PyExc_TypeError, "rows are wanted");
  if (PyErr_Occurred() || group_ints(a[2], y->rows, &n) || i32(a[4], &l->activation) || i32(a[5], &l->type) || as_ptr(a[7], &st)) return -1;
  y->groups = n;
  l->groups = n > PS_MAX_WORKERS ? PS_MAX_WORKERS + 1 : (int32_t)n;      /* more than that the library refuses */
  l->rows = y->rows;
  y->total = 0;
  for (Py_ssize_t i = 0; i < n && i < PS_MAX_WORKERS; ++i) y->total += y->rows[i];
  if (view(a[1], "weight", &w)) return -1;
  if (w.dims < 2) { PyErr_SetString(PyExc_ValueError, "weight: [n_weights, out_features, in_features] is wanted"); return -1; }
  const Py_ssize_t count = w.dims == 3 ? w.size[0] : 1, N = w.size[w.dims - 2], K = w.size[w.dims - 1];
  if (count > INT32_MAX || N > INT32_MAX || K > INT32_MAX) { PyErr_SetString(PyExc_ValueError, "weight is too large"); return -1; }
  l->n_weights = (int32_t)count;
  l->out_features = (int32_t)N;
  l->in_features = (int32_t)K;
  if (a[3] != Py_None) {
    if (group_ints(a[3], y->weights, &nw)) return -1;
    if (nw != n) { PyErr_SetString(PyExc_ValueError, "weight_of: one snapshot per group is wanted"); return -1; }
    l->weight_of = y->weights;
  } else if (n != count) {
    PyErr_SetString(PyExc_ValueError, "weight_of is wanted where the groups are not as many as the weights");
    return -1;
  }
  if (!(y->dtype = PyObject_GetAttr(a[0], n_dtype))) return -1;
  Py_DECREF(y->dtype);
  if (rows_of(a[0], "x", y->total < 0 ? 0 : y->total, K, y->dtype, 0, y->device, &p, &l->x_pitch, NULL)) return -1;
  l->x = p;
  if (stack_of(a[1], "weight", count, N, K, y->dtype, 0, y->device, &p, &l->weight_pitch, &l->weight_stride, NULL)) return -1;
  l->weight = p;
  l->stream = st;
  return 0;
}
/* The workspace, where the tile copies cannot read an operand as it lies. */
static int workspace(PyObject* device, Layer* y, const void* dy, int64_t dy_pitch) {
  ps_dense_layer* l = &y->l;
  if (!((((uintptr_t)l->x | (uintptr_t)l->weight | (uintptr_t)dy) & 15) | ((l->x_pitch | l->weight_pitch | l->weight_stride | dy_pitch) & 7))) return 0;
  uint64_t need = 0;
  if (f_dense_workspace(l, dy, dy_pitch, &need) || !need) return 0;      /* a call that is refused here is refused again where it is made */
  if (!(y->space = PyObject_CallFunction(allocate, "KO", (unsigned long long)need, device))) return -1;
  PyObject* ptr = PyObject_CallMethodNoArgs(y->space, n_data_ptr);
  if (!ptr) { Py_CLEAR(y->space); return -1; }
  l->workspace = PyLong_AsVoidPtr(ptr);
  l->workspace_bytes = need;
  Py_DECREF(ptr);
  return 0;
}

/* (layer..., bias, residual, y, y_type, pre) */
static PyObject* dense_forward(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(LAYER_ARGS + 5)
  Layer y;
  ps_dense_output o;
  void *bias, *residual;
  int64_t unused;
  if (layer(a, &y)) return NULL;
  PyObject* const* b = a + LAYER_ARGS;
  const int64_t M = y.total, N = y.l.out_features;
  memset(&o, 0, sizeof(o));
  if (stack_of(b[0], "bias", y.l.n_weights, -1, N, y.dtype, 0, y.device, &bias, &unused, &o.bias_stride, NULL) ||
      rows_of(b[1], "residual", M, N, y.dtype, 0, y.device, &residual, &o.residual_pitch, NULL) ||
      rows_of(b[2], "y", M, N, y.dtype, 1, y.device, &o.y, &o.y_pitch, NULL) || i32(b[3], &o.y_type) ||
      rows_of(b[4], "pre", M, N, y.dtype, 0, y.device, &o.pre, &o.pre_pitch, NULL) || workspace(a[6], &y, NULL, 0))
    return NULL;
  o.bias = bias;
  o.residual = residual;
  int32_t rc;
  CALL(f_dense_forward(&y.l, &o))
  Py_XDECREF(y.space);
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* (layer..., dy, dx_add, x_pre, dx, dx_pre, dw, db, accumulate) */
static PyObject* dense_backward(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(LAYER_ARGS + 8)
  Layer y;
  ps_dense_gradients o;
  void *dy, *add, *pre;
  int64_t unused;
  PyObject *dw_type = NULL, *db_type = NULL;
  if (layer(a, &y)) return NULL;
  PyObject* const* b = a + LAYER_ARGS;
  const int64_t M = y.total, N = y.l.out_features, K = y.l.in_features;
  memset(&o, 0, sizeof(o));
  if (rows_of(b[0], "dy", M, N, y.dtype, 0, y.device, &dy, &o.dy_pitch, NULL) || rows_of(b[1], "dx_add", M, K, y.dtype, 0, y.device, &add, &o.dx_add_pitch, NULL) ||
      rows_of(b[2], "x_pre", M, K, y.dtype, 0, y.device, &pre, &o.x_pre_pitch, NULL) || rows_of(b[3], "dx", M, K, y.dtype, 0, y.device, &o.dx, &o.dx_pitch, NULL) ||
      rows_of(b[4], "dx_pre", M, K, y.dtype, 0, y.device, &o.dx_pre, &o.dx_pre_pitch, NULL) ||
      stack_of(b[5], "dw", y.groups, N, K, y.dtype, 1, y.device, &o.dw, &o.dw_pitch, &o.dw_stride, &dw_type) ||
      stack_of(b[6], "db", y.groups, -1, N, y.dtype, 1, y.device, &o.db, &unused, &o.db_stride, &db_type) || i32(b[7], &o.accumulate))
    return NULL;
  if (dw_type && db_type && dw_type != db_type) { PyErr_SetString(PyExc_ValueError, "dw and db of one type are wanted"); return NULL; }
  if (workspace(a[6], &y, dy, o.dy_pitch)) return NULL;
  o.dy = dy;
  o.dx_add = add;
  o.x_pre = pre;
  o.dw_type = (dw_type ? dw_type : db_type) == t_float32 ? PS_TYPE_FP32 : y.l.type;
  int32_t rc;
  CALL(f_dense_backward(&y.l, &o))
  Py_XDECREF(y.space);
  if (rc) return raise(rc);
  Py_RETURN_NONE;
}

/* (torch.float32, allocate) */
static PyObject* bind_torch(PyObject* m, PyObject* const* a, Py_ssize_t nargs) {
  WANT(2)
  Py_INCREF(a[0]);
  Py_XSETREF(t_float32, a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(allocate, a[1]);
  Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {FAST(bind), FAST(pull), FAST(reserve), FAST(grad_step), FAST(grad_step_summed), FAST(eval),
                                FAST(enqueue), FAST(apply), FAST(apply_stale), FAST(apply_summed), FAST(apply_adamw), FAST(adamw_step),
                                FAST(dense_forward), FAST(dense_backward), FAST(bind_torch), {NULL, NULL, 0, NULL}};
static struct PyModuleDef def = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  k_applied = PyUnicode_InternFromString("applied");
  k_version = PyUnicode_InternFromString("new_version");
  k_checkpointed = PyUnicode_InternFromString("checkpointed");
  k_replicated = PyUnicode_InternFromString("replicated");
  n_shape = PyUnicode_InternFromString("shape");
  n_stride = PyUnicode_InternFromString("stride");
  n_data_ptr = PyUnicode_InternFromString("data_ptr");
  n_dtype = PyUnicode_InternFromString("dtype");
  n_get_device = PyUnicode_InternFromString("get_device");
  return PyModule_Create(&def);
}
