/* Argument marshalling of the history and node-table operators for Python, without ctypes: checks of the tensors, then the call of the C entry
 * point.  A call through ctypes spends 10 us on twenty arguments, more than its kernels take on small batches; here a tensor costs 0.2 us.
 * Plain CPython API; tensors are asked through their own methods, so nothing is linked against torch.
 *
 * Every function takes its tensors and numbers in the entry point's order and returns None, or (code, message) where the library refuses
 * the call, or the index of the device that has to be made current first.  What is no tensor of the expected kind raises TypeError. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/tgnn.h"

static PyObject *s_dtype, *s_get_device, *s_is_contiguous, *s_numel, *s_data_ptr, *s_size, *s_dim, *s_stride;
enum { I32, I64, F32, F64, BF16, F16, KINDS, U8 = KINDS, I8, ALL };
static PyObject* g_dtype[ALL];
static const char* const g_name[ALL] = {"int32", "int64", "float32", "float64", "bfloat16", "float16", "uint8", "int8"};
static PyObject *g_device, *g_stream;

static struct {
  int (*sample_window)(const int64_t*, const int32_t*, const int32_t*, const double*, int64_t, int64_t, const int32_t*, const double*, int64_t,
                       int, int, int32_t*, int32_t*, double*, int32_t*, int64_t*, int32_t*, int32_t*, void*, char*, int64_t);
  int (*cache_write)(const tgnn_cache*, const void*, int, int64_t, int64_t, const void*, const void*, int, int64_t, const double*, int32_t*,
                     void*, char*, int64_t);
  int (*cache_read)(const tgnn_cache*, void*, int, int64_t, int64_t, const void*, const void*, int, int64_t, double*, int32_t*, void*, char*,
                    int64_t);
  int (*cached_attend)(const void*, int, const tgnn_cache*, const tgnn_cache*, int64_t, int, const int64_t*, const int32_t*, const float*,
                       int, const double*, const double*, const double*, int, int, int, float, void*, int32_t*, void*, char*, int64_t);
  int (*slot_attend)(const void*, const void*, const void*, int, int64_t, int, int, int, int, const int32_t*, const float*, int, const double*,
                     const double*, const double*, float, void*, void*, char*, int64_t);
  int64_t (*slot_attend_scratch)(int64_t, int, int);
  int (*slot_attend_backward)(const void*, const void*, const void*, int, int64_t, int, int, int, int, const int32_t*, const float*, int,
                              const double*, const double*, const double*, float, const void*, void*, void*, void*, float*, float*, void*,
                              char*, int64_t);
} fn;

/* t.name() or t.name(i) as an integer.  -1 where t has no such thing, or one that gives no number (what needed it then raises TypeError), and where it
 * raises: that exception stays, and nothing is asked after it but for the caller to see it (failed() looks, at answers below 0 only). */
static long long integer(PyObject* r) {
  const long long v = !r ? -1 : r == Py_True ? 1 : r == Py_False ? 0 : PyLong_AsLongLong(r);
  Py_XDECREF(r);
  if (v == -1 && PyErr_Occurred() && (PyErr_ExceptionMatches(PyExc_AttributeError) || PyErr_ExceptionMatches(PyExc_TypeError))) PyErr_Clear();
  return v;
}
static int failed(long long v) { return v < 0 && PyErr_Occurred(); }
static long long ask(PyObject* t, PyObject* name) { return integer(PyObject_CallMethodNoArgs(t, name)); }
static long long ask1(PyObject* t, PyObject* name, long i) {
  PyObject* arg = PyLong_FromLong(i);
  if (!arg) return -1;
  const long long v = integer(PyObject_CallMethodOneArg(t, name, arg));
  Py_DECREF(arg);
  return v;
}
static int kind_of(PyObject* t) { /* -1: of no kind that is used here, or no tensor at all */
  PyObject* d = PyObject_GetAttr(t, s_dtype);
  if (!d) {
    if (PyErr_ExceptionMatches(PyExc_AttributeError)) PyErr_Clear();
    return -1;
  }
  Py_DECREF(d); /* dtypes live as long as the interpreter */
  for (int k = 0; k < ALL; ++k)
    if (d == g_dtype[k]) return k;
  return -1;
}
static int is_row(int kind) { return kind == F32 || kind == BF16 || kind == F16; }
static int row_type(int kind) { return kind == F32 ? TGNN_F32 : kind == BF16 ? TGNN_BF16 : TGNN_F16; }

static int refuse(PyObject* t, const char* name, const char* want, long long n, long long dev) { /* an exception that is there stays */
  if (PyErr_Occurred()) return -1;
  const long long has = n >= 0 ? ask(t, s_numel) : 0;
  if (failed(has)) return -1;
  if (n >= 0) PyErr_Format(PyExc_TypeError, "%s: expected a contiguous %s tensor of %lld elements on CUDA device %lld, got %lld in a %s", name,
                           want, n, dev, has, Py_TYPE(t)->tp_name);
  else PyErr_Format(PyExc_TypeError, "%s: expected a %s tensor on a CUDA device, got a %s", name, want, Py_TYPE(t)->tp_name);
  return -1;
}
static int refuse_vec(PyObject* t, const char* name, int kind, long long n, int at_least, long long dev) {
  if (!at_least || PyErr_Occurred()) return refuse(t, name, g_name[kind], n, dev);
  PyErr_Format(PyExc_TypeError, "%s: expected a contiguous %s tensor of at least %lld elements on CUDA device %lld, got a %s", name, g_name[kind], n, dev,
               Py_TYPE(t)->tp_name);
  return -1;
}

/* t.data_ptr(), which a tensor without storage raises for */
static int address(PyObject* t, const char* name, void** out) {
  const long long v = ask(t, s_data_ptr);
  if (v == -1) { /* no tensor lies there */
    if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "%s: a %s has no address", name, Py_TYPE(t)->tp_name);
    return -1;
  }
  *out = (void*)(uintptr_t)v;
  return 0;
}

/* Address of a contiguous tensor on the device of n elements, or at least n; *has = how many there are.  None -> NULL and -1.  -1: refused. */
static int vec_n(PyObject* t, int kind, long long dev, long long n, int at_least, const char* name, void* out, long long* has) {
  void** p = (void**)out;
  *p = NULL;
  *has = -1;
  if (t == Py_None) return 0;
  if (kind_of(t) != kind || ask(t, s_get_device) != dev || ask(t, s_is_contiguous) != 1) return refuse_vec(t, name, kind, n, at_least, dev);
  *has = ask(t, s_numel);
  if (*has < 0 || (at_least ? *has < n : *has != n)) return refuse_vec(t, name, kind, n, at_least, dev);
  return address(t, name, p);
}
static int vec(PyObject* t, int kind, long long dev, long long n, int at_least, const char* name, void* out) {
  long long has;
  return vec_n(t, kind, dev, n, at_least, name, out, &has);
}

/* The current stream of device dev, if it is the current device: 1; another one is current: 0; an exception is set: -1 */
static int stream_of(long long dev, void** out) {
  PyObject* d = PyObject_CallNoArgs(g_device);
  if (!d) return -1;
  const long long cur = PyLong_AsLongLong(d);
  if (cur != dev) {
    Py_DECREF(d);
    return 0;
  }
  PyObject* s = PyObject_CallOneArg(g_stream, d);
  Py_DECREF(d);
  if (!s) return -1;
  *out = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return PyErr_Occurred() ? -1 : 1;
}
static PyObject* result(int rc, const char* err) {
  if (rc == TGNN_OK) Py_RETURN_NONE;
  return Py_BuildValue("(is)", rc, err);
}
#define STREAM(dev)                                            \
  void* stream;                                                \
  char err[512] = "";                                          \
  {                                                            \
    const int st = stream_of(dev, &stream);                    \
    if (st < 0) return NULL;                                   \
    if (st == 0) return PyLong_FromLongLong(dev);              \
  }
/* The library's call, with the interpreter free for other threads (a launch may wait for a full queue or for a module's first loading); the caller
 * holds the tensors meanwhile. */
#define CALL(call)       \
  int rc;                \
  Py_BEGIN_ALLOW_THREADS \
  rc = call;             \
  Py_END_ALLOW_THREADS   \
  return result(rc, err)
#define ARGS(n)                                                                    \
  if (nargs != (n)) return PyErr_Format(PyExc_TypeError, "expected %d arguments", n)
static int number(PyObject* o, long long* v) {
  *v = PyLong_AsLongLong(o);
  return *v == -1 && PyErr_Occurred() ? -1 : 0;
}
static int small(PyObject* o, int* v) { /* an int of the C interface */
  long long x;
  if (number(o, &x)) return -1;
  if (x > INT32_MAX || x < INT32_MIN) {
    PyErr_SetString(PyExc_OverflowError, "a size is beyond int32");
    return -1;
  }
  *v = (int)x;
  return 0;
}
static int shape(PyObject* t, int dims, long long* out, const char* name) {
  if (ask(t, s_dim) != dims) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "%s: expected a tensor of %d dimensions", name, dims);
    return -1;
  }
  for (int i = 0; i < dims; ++i) {
    out[i] = ask1(t, s_size, i);
    if (failed(out[i])) return -1;
  }
  return 0;
}
static int sizes_fit(const long long* v, int n) {
  for (int i = 0; i < n; ++i)
    if (v[i] > INT32_MAX) {
      PyErr_SetString(PyExc_OverflowError, "a size is beyond int32");
      return -1;
    }
  return 0;
}

/* indptr, nbr, eid, ts, nodes, times, window, sinks, nbr_out, eid_out, ts_out, cnt_out, first_out, len_out, status */
static PyObject* py_sample_window(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(15);
  int64_t *indptr, *first;
  int32_t *nbr, *eid, *nodes, *o_nbr, *o_eid, *cnt, *len, *status;
  double *ts, *times, *o_ts;
  int window, sinks;
  const long long dev = ask(a[3], s_get_device);
  if (dev < 0) return refuse(a[3], "ts", "float64", -1, 0), NULL;
  long long n, P, N;
  if (small(a[6], &window) || small(a[7], &sinks) || vec_n(a[0], I64, dev, 1, 1, "indptr", &indptr, &N) ||
      vec_n(a[3], F64, dev, 0, 1, "ts", &ts, &P) || vec_n(a[4], I32, dev, 0, 1, "nodes", &nodes, &n))
    return NULL;
  --N; /* nodes */
  const long long S = n * ((long long)window + sinks);
  if (vec(a[1], I32, dev, P, 0, "nbr", &nbr) || vec(a[2], I32, dev, P, 0, "eid", &eid) || vec(a[5], F64, dev, n, 0, "times", &times) ||
      vec(a[8], I32, dev, S, 0, "nbr_out", &o_nbr) || vec(a[9], I32, dev, S, 0, "eid_out", &o_eid) ||
      vec(a[10], F64, dev, S, 0, "ts_out", &o_ts) || vec(a[11], I32, dev, n, 0, "cnt_out", &cnt) ||
      vec(a[12], I64, dev, n, 0, "first_out", &first) || vec(a[13], I32, dev, n, 0, "len_out", &len) ||
      vec(a[14], I32, dev, 1, 0, "status", &status))
    return NULL;
  STREAM(dev);
  CALL(fn.sample_window(indptr, nbr, eid, ts, N, P, nodes, times, n, window, sinks, o_nbr, o_eid, o_ts, cnt, first, len, status, stream,
       err, sizeof err));
}

/* write, cache address, device, cache rows, heads, dim, rows, status, src, dst, times */
static PyObject* py_cache_move(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(11);
  const int write = a[0] == Py_True;
  const tgnn_cache* c = (const tgnn_cache*)PyLong_AsVoidPtr(a[1]);
  long long dev, cache_rows, heads, dim, stride;
  if (number(a[2], &dev) || number(a[3], &cache_rows) || number(a[4], &heads) || number(a[5], &dim)) return NULL;
  PyObject* rows = a[6];
  const int kind = kind_of(rows);
  if (!is_row(kind) || ask(rows, s_get_device) != dev) return refuse(rows, "rows", "float32, bfloat16 or float16", -1, dev), NULL;
  const long long d = ask(rows, s_dim), num = d < 1 ? -1 : ask1(rows, s_size, 0);
  if (failed(num)) return NULL;
  if (!(d == 2 && ask1(rows, s_size, 1) == heads * dim) && !(d == 3 && ask1(rows, s_size, 1) == heads && ask1(rows, s_size, 2) == dim)) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "rows: expected rows of %lld x %lld values", heads, dim);
    return NULL;
  }
  const long long dense = ask(rows, s_is_contiguous);
  stride = heads * dim;
  if (dense != 1) { /* rows apart, the values of one side by side */
    if (PyErr_Occurred()) return NULL;
    long long s1, s2 = 1;
    if (failed(s1 = ask1(rows, s_stride, 1)) || (d == 3 && failed(s2 = ask1(rows, s_stride, 2)))) return NULL;
    const int inner = d == 2 ? s1 == 1 || stride == 1 : (s1 == dim || heads == 1) && (s2 == 1 || dim == 1);
    if (num > 1) stride = ask1(rows, s_stride, 0);
    if (PyErr_Occurred()) return NULL;
    if (!inner || stride < heads * dim) {
      PyErr_SetString(PyExc_TypeError, "rows: a row's values must lie side by side and rows apart");
      return NULL;
    }
  }
  long long n = write ? num : cache_rows;
  void* idx[2];
  int bits = 64;
  long long count[2] = {-1, -1};
  int kinds[2] = {-1, -1};
  for (int i = 0; i < 2; ++i) {
    PyObject* t = a[8 + i];
    idx[i] = NULL;
    if (t == Py_None) continue;
    kinds[i] = kind_of(t);
    if (kinds[i] != I32 && kinds[i] != I64) return refuse(t, i ? "dst" : "src", "int32 or int64", -1, dev), NULL;
    if (vec_n(t, kinds[i], dev, 0, 1, i ? "dst" : "src", &idx[i], &count[i])) return NULL;
    n = count[i];
    bits = kinds[i] == I64 ? 64 : 32;
  }
  if (kinds[0] >= 0 && kinds[1] >= 0 && (kinds[0] != kinds[1] || count[0] != count[1])) {
    PyErr_SetString(PyExc_TypeError, "src and dst: expected the same type and number of indices");
    return NULL;
  }
  double* times;
  int32_t* status;
  void* p;
  if (address(rows, "rows", &p) || vec(a[10], F64, dev, num, 0, "times", &times) || vec(a[7], I32, dev, 1, 0, "status", &status)) return NULL;
  STREAM(dev);
  CALL((write ? fn.cache_write(c, p, row_type(kind), num, stride, idx[0], idx[1], bits, n, times, status, stream, err, sizeof err)
              : fn.cache_read(c, p, row_type(kind), num, stride, idx[0], idx[1], bits, n, times, status, stream, err, sizeof err)));
}

struct bias {
  float* table;
  double *bounds, *times, *ts;
  int buckets;
};
/* bias, bounds, times, ts */
static int bias_args(PyObject* const* a, long long dev, long long heads, long long n, long long entries, struct bias* b) {
  memset(b, 0, sizeof *b);
  if (a[0] == Py_None) return 0;
  long long sh[2];
  if (shape(a[0], 2, sh, "bias") || sizes_fit(sh, 2)) return -1;
  if (sh[0] != heads) {
    PyErr_Format(PyExc_TypeError, "bias: expected [heads = %lld, buckets]", heads);
    return -1;
  }
  if (a[2] == Py_None || a[3] == Py_None || (a[1] == Py_None && sh[1] > 1)) {
    PyErr_SetString(PyExc_TypeError, "a bias needs bounds, times and ts");
    return -1;
  }
  b->buckets = (int)sh[1];
  return vec(a[0], F32, dev, heads * sh[1], 0, "bias", &b->table) || vec(a[1], F64, dev, sh[1] - 1, 0, "bounds", &b->bounds) ||
                 vec(a[2], F64, dev, n, 0, "times", &b->times) || vec(a[3], F64, dev, entries, 1, "ts", &b->ts)
             ? -1
             : 0;
}

/* k address, v address, device, cache rows, dim, q, first, length, window, sinks, max_len, scale or None, out, status, bias, bounds, times, ts */
static PyObject* py_cached_attend(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(18);
  const tgnn_cache *k = (const tgnn_cache*)PyLong_AsVoidPtr(a[0]), *v = (const tgnn_cache*)PyLong_AsVoidPtr(a[1]);
  long long dev, rows, dim, sh[3];
  int window, sinks, max_len;
  if (number(a[2], &dev) || number(a[3], &rows) || number(a[4], &dim) || small(a[8], &window) || small(a[9], &sinks) || small(a[10], &max_len))
    return NULL;
  const int kind = kind_of(a[5]);
  if (!is_row(kind)) return refuse(a[5], "q", "float32, bfloat16 or float16", -1, dev), NULL;
  if (shape(a[5], 3, sh, "q") || sizes_fit(sh + 1, 2)) return NULL;
  if (sh[2] != dim) return PyErr_Format(PyExc_TypeError, "q: expected [n, heads, dim = %lld]", dim);
  const long long n = sh[0];
  void *q, *out;
  int64_t* first;
  int32_t *len, *status;
  struct bias b;
  const double scale = a[11] == Py_None ? 0.0 : PyFloat_AsDouble(a[11]);
  if (PyErr_Occurred() || vec(a[5], kind, dev, n * sh[1] * dim, 0, "q", &q) || vec(a[12], kind, dev, n * sh[1] * dim, 0, "out", &out) ||
      vec(a[6], I64, dev, n, 0, "first", &first) || vec(a[7], I32, dev, n, 0, "length", &len) || vec(a[13], I32, dev, 1, 0, "status", &status) ||
      bias_args(a + 14, dev, sh[1], n, rows, &b))
    return NULL;
  STREAM(dev);
  const float s = (float)(a[11] == Py_None ? 1.0 / __builtin_sqrt((double)dim) : scale);
  CALL(fn.cached_attend(q, row_type(kind), k, v, n, (int)sh[1], first, len, b.table, b.buckets, b.bounds, b.times, b.ts, window, sinks,
       max_len, s, out, status, stream, err, sizeof err));
}

struct slots {
  void *q, *k, *v;
  int32_t* cnt;
  struct bias b;
  long long dev, n, rows, values;
  int kind, slots, heads, kv, dim;
  float scale;
};
/* q, k, v, cnt, scale or None, bias, bounds, times, ts */
static int slot_args(PyObject* const* a, struct slots* s) {
  long long sh[3], rw[4];
  s->kind = kind_of(a[0]);
  s->dev = !is_row(s->kind) ? -1 : ask(a[0], s_get_device);
  if (s->dev < 0) return refuse(a[0], "q", "float32, bfloat16 or float16", -1, 0);
  if (shape(a[0], 3, sh, "q") || shape(a[1], 4, rw, "k") || sizes_fit(sh + 1, 2) || sizes_fit(rw + 1, 2)) return -1;
  if (rw[0] != sh[0] || rw[3] != sh[2]) {
    PyErr_SetString(PyExc_TypeError, "expected q [n, heads, dim] and k [n, slots, kv_heads, dim]");
    return -1;
  }
  s->n = sh[0];
  s->heads = (int)sh[1];
  s->dim = (int)sh[2];
  s->slots = (int)rw[1];
  s->kv = (int)rw[2];
  s->values = sh[0] * sh[1] * sh[2];
  s->rows = rw[0] * rw[1] * rw[2] * rw[3];
  const double scale = a[4] == Py_None ? 1.0 / __builtin_sqrt((double)s->dim) : PyFloat_AsDouble(a[4]);
  s->scale = (float)scale;
  return PyErr_Occurred() || vec(a[0], s->kind, s->dev, s->values, 0, "q", &s->q) || vec(a[1], s->kind, s->dev, s->rows, 0, "k", &s->k) ||
                 vec(a[2], s->kind, s->dev, s->rows, 0, "v", &s->v) || vec(a[3], I32, s->dev, s->n, 0, "cnt", &s->cnt) ||
                 bias_args(a + 5, s->dev, s->heads, s->n, s->n * s->slots, &s->b)
             ? -1
             : 0;
}

/* q, k, v, cnt, scale, bias, bounds, times, ts, out */
static PyObject* py_slot_attend(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(10);
  struct slots s;
  void* out;
  if (slot_args(a, &s) || vec(a[9], s.kind, s.dev, s.values, 0, "out", &out)) return NULL;
  STREAM(s.dev);
  CALL(fn.slot_attend(s.q, s.k, s.v, row_type(s.kind), s.n, s.slots, s.heads, s.kv, s.dim, s.cnt, s.b.table, s.b.buckets, s.b.bounds,
       s.b.times, s.b.ts, s.scale, out, stream, err, sizeof err));
}

/* q, k, v, cnt, scale, bias, bounds, times, ts, dout, dq, dk, dv, dbias, scratch */
static PyObject* py_slot_attend_backward(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(15);
  struct slots s;
  void *dout, *dq, *dk, *dv;
  float *dbias, *scratch = NULL;
  if (slot_args(a, &s)) return NULL;
  if ((a[5] == Py_None) != (a[13] == Py_None) || (a[13] != Py_None && a[14] == Py_None)) {
    PyErr_SetString(PyExc_TypeError, "dbias and scratch belong to a bias");
    return NULL;
  }
  if (vec(a[9], s.kind, s.dev, s.values, 0, "dout", &dout) || vec(a[10], s.kind, s.dev, s.values, 0, "dq", &dq) ||
      vec(a[11], s.kind, s.dev, s.rows, 0, "dk", &dk) || vec(a[12], s.kind, s.dev, s.rows, 0, "dv", &dv) ||
      vec(a[13], F32, s.dev, (long long)s.heads * s.b.buckets, 0, "dbias", &dbias))
    return NULL;
  if (a[13] != Py_None) {
    const long long need = fn.slot_attend_scratch(s.n, s.heads, s.b.buckets);
    if (vec(a[14], F32, s.dev, need < 0 ? 0 : need, 1, "scratch", &scratch)) return NULL;
  }
  STREAM(s.dev);
  CALL(fn.slot_attend_backward(s.q, s.k, s.v, row_type(s.kind), s.n, s.slots, s.heads, s.kv, s.dim, s.cnt, s.b.table, s.b.buckets,
       s.b.bounds, s.b.times, s.b.ts, s.scale, dout, dq, dk, dv, dbias, scratch, stream, err, sizeof err));
}

/* (dtypes in the order of the enumeration), current device's and current stream's callables, (addresses of the entry points) */
static PyObject* py_init(PyObject* self, PyObject* args) {
  PyObject *dt, *at;
  if (!PyArg_ParseTuple(args, "O!OOO!", &PyTuple_Type, &dt, &g_device, &g_stream, &PyTuple_Type, &at)) return NULL;
  if (PyTuple_GET_SIZE(dt) != KINDS || PyTuple_GET_SIZE(at) * sizeof(void*) != sizeof fn)
    return PyErr_Format(PyExc_TypeError, "expected %d dtypes and %d addresses", (int)KINDS, (int)(sizeof fn / sizeof(void*)));
  Py_INCREF(g_device);
  Py_INCREF(g_stream);
  for (int k = 0; k < KINDS; ++k) Py_INCREF(g_dtype[k] = PyTuple_GET_ITEM(dt, k));
  void* p[sizeof fn / sizeof(void*)];
  for (size_t i = 0; i < sizeof fn / sizeof(void*); ++i) p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(at, i));
  if (PyErr_Occurred()) return NULL;
  memcpy(&fn, p, sizeof fn);
  Py_RETURN_NONE;
}

/* ---- node-table operators ---- */
static struct {
  int (*lookup)(const void*, int, int64_t, int, const void*, int, int64_t, float, void*, int, int32_t*, void*, char*, int64_t);
  int64_t (*lookup_scratch)(int64_t, int64_t, int);
  int (*lookup_backward)(const void*, int, int64_t, const void*, int, int64_t, int, float, void*, int, void*, int32_t*, void*, char*, int64_t);
  int64_t (*loss_kept)(int64_t, int);
  int64_t (*loss_scratch)(int64_t, int64_t, int, int);
  int (*loss)(const void*, const void*, int, int64_t, int64_t, int, const void*, int, const float*, float, float*, float*, void*, int32_t*, void*,
              char*, int64_t);
  int (*loss_backward)(const void*, const void*, int, int64_t, int64_t, int, const void*, int, const float*, float, const float*, const float*, void*,
                       void*, float*, void*, int32_t*, void*, char*, int64_t);
  int (*adamw_step)(const tgnn_adamw_tensor*, int, int, int64_t*, double, double, double, double, double, uint64_t, void*, char*, int64_t);
  int (*adamw_moments)(const tgnn_adamw_tensor*, int, float* const*, float* const*, void*, char*, int64_t);
} table_fn;

/* A dense 2D tensor of rows of any row type; dev < 0: on any device */
static int matrix(PyObject* t, long long* dev, const char* name, int* kind, long long* sh, void** p) {
  *kind = kind_of(t);
  const long long on = !is_row(*kind) ? -1 : ask(t, s_get_device);
  if (on < 0 || (*dev >= 0 && on != *dev)) return refuse(t, name, "float32, bfloat16 or float16", -1, *dev);
  *dev = on;
  if (shape(t, 2, sh, name) || sizes_fit(sh + 1, 1)) return -1;
  return vec(t, *kind, on, sh[0] * sh[1], 0, name, p);
}
static int indices(PyObject* t, long long dev, const char* name, int* bits, long long* n, void** p) {
  const int kind = kind_of(t);
  if (kind != I32 && kind != I64) return refuse(t, name, "int32 or int64", -1, dev);
  *bits = kind == I64 ? 64 : 32;
  return vec_n(t, kind, dev, 0, 1, name, p, n);
}
/* rows of any row type, n * dim values in any shape */
static int rows_of(PyObject* t, long long dev, long long values, const char* name, int* kind, void** p) {
  *kind = kind_of(t);
  if (!is_row(*kind)) return refuse(t, name, "float32, bfloat16 or float16", -1, dev);
  return vec(t, *kind, dev, values, 0, name, p);
}
static int scratch_of(PyObject* t, long long dev, long long need, void** p) {
  if (t == Py_None) {
    PyErr_SetString(PyExc_TypeError, "scratch: expected a uint8 tensor");
    return -1;
  }
  return vec(t, U8, dev, need < 0 ? 0 : need, 1, "scratch", p);
}
static int must(PyObject* t, const char* name) {
  if (t != Py_None) return 0;
  PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got None", name);
  return -1;
}

/* table, ids, out, scale, status */
static PyObject* py_lookup(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(5);
  long long dev = -1, sh[2], n;
  int kind, out_kind, bits;
  void *table, *ids, *out;
  int32_t* status;
  const double scale = PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred() || matrix(a[0], &dev, "table", &kind, sh, &table) || indices(a[1], dev, "ids", &bits, &n, &ids) ||
      rows_of(a[2], dev, n * sh[1], "out", &out_kind, &out) || must(a[4], "status") || vec(a[4], I32, dev, 1, 0, "status", &status))
    return NULL;
  STREAM(dev);
  CALL(table_fn.lookup(table, row_type(kind), sh[0], (int)sh[1], ids, bits, n, (float)scale, out, row_type(out_kind), status, stream, err, sizeof err));
}

/* ids, dout, dtable, scratch, scale, status */
static PyObject* py_lookup_backward(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(6);
  long long dev = -1, sh[2], n;
  int kind, out_kind, bits;
  void *dtable, *ids, *dout, *scratch;
  int32_t* status;
  const double scale = PyFloat_AsDouble(a[4]);
  if (PyErr_Occurred() || matrix(a[2], &dev, "dtable", &kind, sh, &dtable) || indices(a[0], dev, "ids", &bits, &n, &ids) ||
      rows_of(a[1], dev, n * sh[1], "dout", &out_kind, &dout) || scratch_of(a[3], dev, table_fn.lookup_scratch(n, sh[0], (int)sh[1]), &scratch) ||
      must(a[5], "status") || vec(a[5], I32, dev, 1, 0, "status", &status))
    return NULL;
  STREAM(dev);
  CALL(table_fn.lookup_backward(ids, bits, n, dout, row_type(out_kind), sh[0], (int)sh[1], (float)scale, dtable, row_type(kind), scratch, status,
       stream, err, sizeof err));
}

struct loss {
  void *q, *table, *target, *scratch;
  float* bias;
  int32_t* status;
  long long dev, n, rows;
  int kind, bits, dim;
  float scale;
};
/* q, table, target, bias, scale or None, scratch, status */
static int loss_args(PyObject* const* a, struct loss* l) {
  long long sh[2], rw[2], n;
  int kind;
  l->dev = -1;
  if (matrix(a[0], &l->dev, "q", &l->kind, sh, &l->q) || matrix(a[1], &l->dev, "table", &kind, rw, &l->table) ||
      indices(a[2], l->dev, "target", &l->bits, &n, &l->target))
    return -1;
  if (kind != l->kind || rw[1] != sh[1] || n != sh[0]) {
    PyErr_SetString(PyExc_TypeError, "expected q [n, dim], table [rows, dim] of one type and target [n]");
    return -1;
  }
  l->n = n;
  l->rows = rw[0];
  l->dim = (int)sh[1];
  const double scale = a[4] == Py_None ? 1.0 / __builtin_sqrt((double)(l->dim < 1 ? 1 : l->dim)) : PyFloat_AsDouble(a[4]);
  l->scale = (float)scale;
  return PyErr_Occurred() || vec(a[3], F32, l->dev, l->rows, 0, "bias", &l->bias) ||
                 scratch_of(a[5], l->dev, table_fn.loss_scratch(l->n, l->rows, l->dim, row_type(l->kind)), &l->scratch) || must(a[6], "status") ||
                 vec(a[6], I32, l->dev, 1, 0, "status", &l->status)
             ? -1
             : 0;
}

/* q, table, target, bias, scale or None, scratch, status, loss, kept */
static PyObject* py_destination_loss(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(9);
  struct loss l;
  float *loss, *kept;
  if (loss_args(a, &l) || must(a[7], "loss") || vec(a[7], F32, l.dev, l.n, 0, "loss", &loss) ||
      vec(a[8], F32, l.dev, table_fn.loss_kept(l.n, l.dim), 0, "kept", &kept))
    return NULL;
  STREAM(l.dev);
  CALL(table_fn.loss(l.q, l.table, row_type(l.kind), l.n, l.rows, l.dim, l.target, l.bits, l.bias, l.scale, loss, kept, l.scratch, l.status, stream,
       err, sizeof err));
}

/* q, table, target, bias, scale or None, scratch, status, kept, dloss, dq, dtable, dbias */
static PyObject* py_destination_loss_backward(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(12);
  struct loss l;
  float *kept, *dloss, *dbias;
  void *dq, *dtable;
  if (loss_args(a, &l) || must(a[7], "kept") || vec(a[7], F32, l.dev, table_fn.loss_kept(l.n, l.dim), 0, "kept", &kept) || must(a[8], "dloss") ||
      vec(a[8], F32, l.dev, l.n, 0, "dloss", &dloss) || vec(a[9], l.kind, l.dev, l.n * l.dim, 0, "dq", &dq) ||
      vec(a[10], l.kind, l.dev, l.rows * l.dim, 0, "dtable", &dtable) || vec(a[11], F32, l.dev, l.rows, 0, "dbias", &dbias))
    return NULL;
  STREAM(l.dev);
  CALL(table_fn.loss_backward(l.q, l.table, row_type(l.kind), l.n, l.rows, l.dim, l.target, l.bits, l.bias, l.scale, kept, dloss, dq, dtable, dbias,
       l.scratch, l.status, stream, err, sizeof err));
}

/* descriptions' address, bits, device, steps, lr, beta1, beta2, eps, grad_scale, seed, params, grads (lists; a gradient may be None) */
static PyObject* py_adamw_step(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(12);
  const tgnn_adamw_tensor* held = (const tgnn_adamw_tensor*)PyLong_AsVoidPtr(a[0]);
  long long dev;
  int bits;
  double x[5];
  int64_t* steps;
  if (small(a[1], &bits) || number(a[2], &dev)) return NULL;
  for (int i = 0; i < 5; ++i) x[i] = PyFloat_AsDouble(a[4 + i]);
  const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[9]);
  if (PyErr_Occurred() || must(a[3], "steps") || vec(a[3], I64, dev, 2, 0, "steps", &steps)) return NULL;
  if (!PyList_Check(a[10]) || !PyList_Check(a[11]) || PyList_GET_SIZE(a[10]) != PyList_GET_SIZE(a[11]))
    return PyErr_Format(PyExc_TypeError, "expected as many gradients as parameters");
  const Py_ssize_t count = PyList_GET_SIZE(a[10]);
  tgnn_adamw_tensor* t = (tgnn_adamw_tensor*)PyMem_Malloc((count ? count : 1) * sizeof *t);
  if (!t) return PyErr_NoMemory();
  memcpy(t, held, count * sizeof *t);
  int bad = 0;
  for (Py_ssize_t i = 0; i < count && !bad; ++i) {
    PyObject* g = PyList_GET_ITEM(a[11], i);
    if (g == Py_None) {
      t[i].numel = 0;
      continue;
    }
    const int kind = kind_of(g);
    if (!is_row(kind)) bad = refuse(g, "grad", "float32, bfloat16 or float16", -1, dev);
    else bad = vec(PyList_GET_ITEM(a[10], i), F32, dev, t[i].numel, 0, "param", &t[i].param) || vec(g, kind, dev, t[i].numel, 0, "grad", &t[i].grad);
    t[i].grad_dtype = row_type(kind);
  }
  void* stream;
  char err[512] = "";
  const int st = bad ? -1 : stream_of(dev, &stream);
  if (st < 1) {
    PyMem_Free(t);
    return st < 0 ? NULL : PyLong_FromLongLong(dev);
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = table_fn.adamw_step(t, (int)count, bits, steps, x[0], x[1], x[2], x[3], x[4], seed, stream, err, sizeof err);
  Py_END_ALLOW_THREADS
  PyMem_Free(t);
  return result(rc, err);
}

/* descriptions' address, count, addresses of the outputs' pointers (m, v), device */
static PyObject* py_adamw_moments(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  ARGS(5);
  const tgnn_adamw_tensor* t = (const tgnn_adamw_tensor*)PyLong_AsVoidPtr(a[0]);
  float *const *m = (float* const*)PyLong_AsVoidPtr(a[2]), *const *v = (float* const*)PyLong_AsVoidPtr(a[3]);
  long long dev;
  int count;
  if (small(a[1], &count) || number(a[4], &dev) || PyErr_Occurred()) return NULL;
  STREAM(dev);
  CALL(table_fn.adamw_moments(t, count, m, v, stream, err, sizeof err));
}

/* (uint8, int8), (addresses of the node-table entry points); after init */
static PyObject* py_init_table(PyObject* self, PyObject* args) {
  PyObject *dt, *at;
  if (!PyArg_ParseTuple(args, "O!O!", &PyTuple_Type, &dt, &PyTuple_Type, &at)) return NULL;
  if (PyTuple_GET_SIZE(dt) != ALL - KINDS || PyTuple_GET_SIZE(at) * sizeof(void*) != sizeof table_fn)
    return PyErr_Format(PyExc_TypeError, "expected %d dtypes and %d addresses", (int)(ALL - KINDS), (int)(sizeof table_fn / sizeof(void*)));
  void* p[sizeof table_fn / sizeof(void*)];
  for (size_t i = 0; i < sizeof table_fn / sizeof(void*); ++i) p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(at, i));
  if (PyErr_Occurred()) return NULL;
  for (int k = KINDS; k < ALL; ++k) Py_INCREF(g_dtype[k] = PyTuple_GET_ITEM(dt, k - KINDS));
  memcpy(&table_fn, p, sizeof table_fn);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"init", py_init, METH_VARARGS, NULL},
                                {"sample_window", (PyCFunction)(void (*)(void))py_sample_window, METH_FASTCALL, NULL},
                                {"cache_move", (PyCFunction)(void (*)(void))py_cache_move, METH_FASTCALL, NULL},
                                {"cached_attend", (PyCFunction)(void (*)(void))py_cached_attend, METH_FASTCALL, NULL},
                                {"slot_attend", (PyCFunction)(void (*)(void))py_slot_attend, METH_FASTCALL, NULL},
                                {"slot_attend_backward", (PyCFunction)(void (*)(void))py_slot_attend_backward, METH_FASTCALL, NULL},
                                {"init_table", py_init_table, METH_VARARGS, NULL},
                                {"lookup", (PyCFunction)(void (*)(void))py_lookup, METH_FASTCALL, NULL},
                                {"lookup_backward", (PyCFunction)(void (*)(void))py_lookup_backward, METH_FASTCALL, NULL},
                                {"destination_loss", (PyCFunction)(void (*)(void))py_destination_loss, METH_FASTCALL, NULL},
                                {"destination_loss_backward", (PyCFunction)(void (*)(void))py_destination_loss_backward, METH_FASTCALL, NULL},
                                {"adamw_step", (PyCFunction)(void (*)(void))py_adamw_step, METH_FASTCALL, NULL},
                                {"adamw_moments", (PyCFunction)(void (*)(void))py_adamw_moments, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  s_dtype = PyUnicode_InternFromString("dtype");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_numel = PyUnicode_InternFromString("numel");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_size = PyUnicode_InternFromString("size");
  s_dim = PyUnicode_InternFromString("dim");
  s_stride = PyUnicode_InternFromString("stride");
  return PyModule_Create(&module);
}
