/*
 * Argument marshalling of the binding's calls that a step makes over and over:
 * reads the tensors' attributes through the Python C API, checks them, and
 * calls the C ABI (include/jfkv.h).  The same checks written in Python take
 * 3.5 to 4 us of a 6.7 us call on a Grace core, here under 2.
 *
 * Uses Python's API alone, no torch headers: a tensor is whatever has dtype,
 * is_cuda, is_contiguous(), data_ptr(), shape and stride().  The functions
 * return the C entry point's status; what is no tensor of the right kind
 * raises TypeError, what does not fit together ValueError.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "jfkv.h"

typedef int (*rows_fn)(const jf_kv_pool*, const int32_t*, int32_t, int32_t, const int32_t*,
                       const int32_t*, void*, int64_t, void*, int64_t, int32_t, int32_t*, void*);

static struct {
  rows_fn append, read;
  int (*rope)(const jf_rope*, const int32_t*, int64_t, int32_t, int32_t, const jf_rope_rows*,
              const jf_rope_rows*, int32_t, int32_t, void*);
  int (*decode)(const jf_kv_pool*, const int32_t*, int32_t, const int32_t*, int32_t, const void*,
                int32_t, float, void*, void*, size_t, int32_t, void*);
  int (*weights)(const jf_kv_pool*, const int32_t*, int32_t, const int32_t*, int32_t, const void*,
                 int32_t, float, void*, const float*, float*, int64_t, void*, size_t, int32_t,
                 void*);
  int (*evict)(const jf_kv_pool*, const int32_t*, int32_t, const int32_t*, int32_t, const float*,
               int64_t, int32_t, int32_t, int32_t, const int32_t*, int32_t, int32_t*, float*,
               int32_t*, int32_t*, void*);
  PyObject *i32, *u8, *f32, *bf16, *f16;      /* torch dtypes */
  PyObject *raw_stream, *get_device;          /* or raw_stream NULL: current_stream */
  PyObject* current_stream;
  PyObject *grad_enabled, *written;           /* torch.is_grad_enabled, autograd's increment_version */
} G;

static PyObject *s_dtype, *s_is_cuda, *s_contig, *s_ptr, *s_shape, *s_stride, *s_numel, *s_stream, *s_grad;
static PyObject *s_data, *s_page, *s_hkv, *s_dim, *s_group, *s_format;

/* ---- tensors ------------------------------------------------------------- */
static int wrong_type(const char* name, const char* what) {
  if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_AttributeError)) return -1;
  PyErr_Clear();
  PyErr_Format(PyExc_TypeError, "%s must be a %s", name, what);
  return -1;
}

static int is_true_attr(PyObject* t, PyObject* name) {
  PyObject* v = PyObject_GetAttr(t, name);
  if (!v) return -1;
  const int r = v == Py_True;
  Py_DECREF(v);
  return r;
}

/* a CUDA tensor of one dtype (checked by identity), contiguous or not -> its pointer */
static int tensor(PyObject* t, PyObject* dtype, const char* name, int contiguous,
                  const char* what, void** ptr) {
  PyObject* d = PyObject_GetAttr(t, s_dtype);
  if (!d) return wrong_type(name, what);
  const int same = d == dtype;
  Py_DECREF(d);
  if (!same || is_true_attr(t, s_is_cuda) != 1) return wrong_type(name, what);
  if (contiguous) {
    PyObject* c = PyObject_CallMethodNoArgs(t, s_contig);
    if (!c) return wrong_type(name, what);
    const int yes = c == Py_True;
    Py_DECREF(c);
    if (!yes) return wrong_type(name, what);
  }
  PyObject* p = PyObject_CallMethodNoArgs(t, s_ptr);
  if (!p) return wrong_type(name, what);
  *ptr = PyLong_AsVoidPtr(p);
  Py_DECREF(p);
  return PyErr_Occurred() ? -1 : 0;
}

#define I32_T "contiguous CUDA tensor of dtype torch.int32"
#define F32_T "contiguous CUDA tensor of dtype torch.float32"
#define BF16_T "contiguous CUDA tensor of dtype torch.bfloat16"
#define U8_T "contiguous CUDA tensor of dtype torch.uint8"

/* shape or stride() into out[4]; the count, -1 on an error, more than 4 counted but not kept */
static int ints_of(PyObject* t, int strides, int64_t* out) {
  PyObject* s = strides ? PyObject_CallMethodNoArgs(t, s_stride) : PyObject_GetAttr(t, s_shape);
  if (!s) return -1;
  int n = -1;
  if (PyTuple_Check(s)) {
    n = (int)PyTuple_GET_SIZE(s);
    for (int i = 0; i < n && i < 4; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
    if (PyErr_Occurred()) n = -1;
  } else {
    PyErr_SetString(PyExc_TypeError, "a tensor's shape is a tuple");
  }
  Py_DECREF(s);
  return n;
}

static int64_t numel(PyObject* t) {
  PyObject* n = PyObject_CallMethodNoArgs(t, s_numel);
  if (!n) return -1;
  const int64_t v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  return v;
}

static int bad(const char* what) {
  PyErr_SetString(PyExc_ValueError, what);
  return -1;
}

static int stream_of(PyObject* stream, void** out) {
  PyObject* h = NULL;
  if (stream == Py_None && G.raw_stream) {
    PyObject* dev = PyObject_CallNoArgs(G.get_device);
    if (!dev) return -1;
    h = PyObject_CallOneArg(G.raw_stream, dev);
    Py_DECREF(dev);
  } else if (stream == Py_None) {
    PyObject* s = PyObject_CallNoArgs(G.current_stream);
    if (!s) return -1;
    h = PyObject_GetAttr(s, s_stream);
    Py_DECREF(s);
  } else if (PyLong_Check(stream)) {
    h = Py_NewRef(stream);
  } else {   /* an object with a handle, or what int() takes */
    h = PyObject_GetAttr(stream, s_stream);
    if (!h && PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      h = PyNumber_Long(stream);
    }
  }
  if (!h) return -1;
  *out = (void*)(uintptr_t)PyLong_AsUnsignedLongLong(h);
  Py_DECREF(h);
  return PyErr_Occurred() ? -1 : 0;
}

static int int_of(PyObject* v, int32_t* out) {
  const long x = PyLong_AsLong(v);
  if (x == -1 && PyErr_Occurred()) return -1;
  if (x < INT32_MIN || x > INT32_MAX) return bad("a size is past 32 bits");
  *out = (int32_t)x;
  return 0;
}

static int int_attr(PyObject* o, PyObject* name, int32_t* out) {
  PyObject* v = PyObject_GetAttr(o, name);
  if (!v) return -1;
  const int r = int_of(v, out);
  Py_DECREF(v);
  return r;
}

/* a pool without a codec */
static int pool_of(PyObject* p, jf_kv_pool* out) {
  PyObject* data = PyObject_GetAttr(p, s_data);
  if (!data) return -1;
  int64_t shape[4] = {0, 0, 0, 0};
  PyObject* at = PyObject_CallMethodNoArgs(data, s_ptr);
  const int n = at ? ints_of(data, 0, shape) : -1;
  Py_DECREF(data);
  if (at) {
    out->base = PyLong_AsVoidPtr(at);
    Py_DECREF(at);
  }
  if (n < 1) return n ? -1 : bad("a pool's data must be [pages, bytes]");
  out->num_pages = shape[0];
  out->tq4 = NULL;
  return int_attr(p, s_page, &out->page_size) || int_attr(p, s_hkv, &out->num_kv_heads) ||
                 int_attr(p, s_dim, &out->head_dim) || int_attr(p, s_group, &out->group_size) ||
                 int_attr(p, s_format, &out->format)
             ? -1
             : 0;
}

static int fit(int64_t n) { return n > INT32_MAX ? bad("a size is past 32 bits") : 0; }

/* the entry point's call, other threads running meanwhile: a launch waits while the queue is full */
#define CALL(call)                \
  do {                            \
    int status;                   \
    Py_BEGIN_ALLOW_THREADS        \
    status = call;                \
    Py_END_ALLOW_THREADS          \
    return PyLong_FromLong(status); \
  } while (0)

static int want(Py_ssize_t n, Py_ssize_t is) {
  if (n == is) return 0;
  PyErr_Format(PyExc_TypeError, "%zd arguments, and %zd are needed", is, n);
  return -1;
}

/* ---- append and read: pool, page_table, start_pos, row_offsets, k, v, err, stream ---- */
static int rows_arg(PyObject* x, const char* name, const jf_kv_pool* p, void** ptr, int64_t* n,
                    int64_t* stride) {
  int64_t sh[4], st[4];
  if (tensor(x, G.bf16, name, 0, "CUDA tensor of dtype torch.bfloat16", ptr)) return -1;
  const int d = ints_of(x, 0, sh);
  if (d < 0) return -1;
  if (d != 3 || sh[1] != p->num_kv_heads || sh[2] != p->head_dim) {
    PyErr_Format(PyExc_ValueError, "%s must be [rows, Hkv, D]", name);
    return -1;
  }
  if (ints_of(x, 1, st) != 3) return -1;
  if (sh[0] && (st[2] != 1 || (sh[1] > 1 && st[1] != sh[2]))) {
    PyErr_Format(PyExc_ValueError, "%s: the elements of a row must adjoin", name);
    return -1;
  }
  *n = sh[0];
  /* the row stride of a single row is whatever a slicing left: it is not used */
  *stride = sh[0] > 1 ? st[0] : sh[1] * sh[2];
  return 0;
}

static PyObject* rows_call(rows_fn fn, PyObject* const* a, Py_ssize_t na) {
  jf_kv_pool p;
  void *pt, *start, *off, *k, *v, *err = NULL, *stream;
  int64_t n, nv, ks, vs, sh[4];
  if (want(8, na) || pool_of(a[0], &p) || tensor(a[1], G.i32, "page_table", 1, I32_T, &pt) ||
      tensor(a[2], G.i32, "start_pos", 1, I32_T, &start) ||
      tensor(a[3], G.i32, "row_offsets", 1, I32_T, &off) || rows_arg(a[4], "k", &p, &k, &n, &ks) ||
      rows_arg(a[5], "v", &p, &v, &nv, &vs) ||
      (a[6] != Py_None && tensor(a[6], G.i32, "err_flag", 1, I32_T, &err)))
    return NULL;
  const int d = ints_of(a[1], 0, sh);
  if (d < 0 || (d == 0 && bad("page_table must be [requests, pages]"))) return NULL;
  const int64_t B = d == 2 ? sh[0] : 1, cols = d == 2 ? sh[1] : numel(a[1]);
  if (n != nv && bad("k and v must have the same rows")) return NULL;
  if ((numel(a[2]) != B || numel(a[3]) != B + 1) &&
      bad("one start_pos per page-table row, and one row offset more"))
    return NULL;
  if (stream_of(a[7], &stream)) return NULL;
  if (fit(cols) || fit(B) || fit(n)) return NULL;
  CALL(fn(&p, pt, (int32_t)cols, (int32_t)B, start, off, k, ks, v, vs, (int32_t)n, err, stream));
}
static PyObject* kv8_append(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  (void)m;
  return rows_call(G.append, a, n);
}
static PyObject* kv8_read(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  (void)m;
  return rows_call(G.read, a, n);
}

/* ---- autograd does not see a call: rows that need a gradient are not written over; those written
 * get a new version, so that a graph that has saved them notices ---- */
static int may_write(PyObject* t, const char* name) {
  const int needs = is_true_attr(t, s_grad);
  if (needs <= 0) return needs;
  PyObject* on = PyObject_CallNoArgs(G.grad_enabled);
  if (!on) return -1;
  const int recorded = on == Py_True;
  Py_DECREF(on);
  if (!recorded) return 0;
  PyErr_Format(PyExc_ValueError, "%s would be written over, and needs a gradient that this call does not record: "
               "give an output, or call it under torch.no_grad()", name);
  return -1;
}
static int was_written(PyObject* q, PyObject* k) {
  PyObject* both = q && k ? PyTuple_Pack(2, q, k) : PyTuple_Pack(1, q ? q : k);
  if (!both) return -1;
  PyObject* r = PyObject_CallOneArg(G.written, both);
  Py_DECREF(both);
  if (!r) return -1;
  Py_DECREF(r);
  return 0;
}

/* ---- rope: address and axes of the handle, positions, q, q_out, k, k_out, inverse, stream ---- */
static int rope_rows(PyObject* x, PyObject* out, const char* name, int64_t n, jf_rope_rows* r,
                     int* dtype, int64_t* dim) {
  *dtype = -1;
  *dim = 0;
  memset(r, 0, sizeof *r);
  if (x == Py_None) return 0;
  int64_t sh[4], st[4], os[4], so[4];
  PyObject* d = PyObject_GetAttr(x, s_dtype);
  if (!d) return wrong_type(name, "CUDA tensor of bf16, fp16 or fp32");
  Py_DECREF(d);   /* the dtypes live as long as torch */
  *dtype = d == G.bf16 ? JF_DTYPE_BF16 : d == G.f16 ? JF_DTYPE_F16 : d == G.f32 ? JF_DTYPE_F32 : -1;
  if (*dtype < 0) return wrong_type(name, "CUDA tensor of bf16, fp16 or fp32");
  void *in, *to;
  if (tensor(x, d, name, 0, "CUDA tensor of bf16, fp16 or fp32", &in)) return -1;
  const int nd = ints_of(x, 0, sh);
  if (nd < 0) return -1;
  if (nd != 3 || sh[0] != n) {
    PyErr_Format(PyExc_ValueError, "%s must be [tokens, heads, head_dim]", name);
    return -1;
  }
  if (ints_of(x, 1, st) != 3) return -1;
  to = in;
  memcpy(os, st, sizeof os);
  if (out != Py_None) {
    if (tensor(out, d, name, 0, "CUDA tensor, and its output one of its dtype", &to)) return -1;
    const int no = ints_of(out, 0, so);
    if (no < 0) return -1;
    if (no != 3 || so[0] != sh[0] || so[1] != sh[1] || so[2] != sh[2]) {
      PyErr_Format(PyExc_ValueError, "%s's output must have its shape", name);
      return -1;
    }
    if (ints_of(out, 1, os) != 3) return -1;
  }
  if (st[2] != 1 || os[2] != 1) {
    PyErr_Format(PyExc_ValueError, "%s: the channels of a head must adjoin", name);
    return -1;
  }
  r->in = in;
  r->out = to;
  r->in_token_stride = st[0];
  r->in_head_stride = st[1];
  r->out_token_stride = os[0];
  r->out_head_stride = os[1];
  if (fit(sh[1]) || may_write(out != Py_None ? out : x, name)) return -1;
  r->num_heads = (int32_t)sh[1];
  *dim = sh[2];
  return 0;
}

static PyObject* rope_axes(PyObject* m, PyObject* const* a, Py_ssize_t na) {
  (void)m;
  void *pos, *stream;
  int64_t sh[4], st[4], qd, kd;
  int qt, kt;
  jf_rope_rows q, k;
  if (want(8, na)) return NULL;
  const jf_rope* rope = PyLong_AsVoidPtr(a[0]);
  if (!rope || tensor(a[1], G.i32, "positions", 0, "CUDA tensor of dtype torch.int32", &pos)) return NULL;
  const int d = ints_of(a[1], 0, sh);
  if (d < 0 || ints_of(a[1], 1, st) != d) return NULL;
  if ((d != 2 || sh[0] != rope->num_axes || (sh[1] > 1 && st[1] != 1)) &&
      bad("positions must be [axes, tokens], the tokens of an axis adjoining"))
    return NULL;
  if (rope_rows(a[2], a[3], "q", sh[1], &q, &qt, &qd) ||
      rope_rows(a[4], a[5], "k", sh[1], &k, &kt, &kd))
    return NULL;
  if (qt < 0 && kt < 0 && bad("q or k is needed")) return NULL;
  if (qt >= 0 && kt >= 0 && (qt != kt || qd != kd) && bad("q and k must have one dtype and head_dim"))
    return NULL;
  const int inverse = PyObject_IsTrue(a[6]);
  if (inverse < 0 || stream_of(a[7], &stream)) return NULL;
  if (fit(sh[1]) || fit(qd) || fit(kd)) return NULL;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = G.rope(rope, pos, st[0], (int32_t)sh[1], (int32_t)(qt >= 0 ? qd : kd), &q, &k,
                  qt >= 0 ? qt : kt, inverse, stream);
  Py_END_ALLOW_THREADS
  if (status == JF_OK && was_written(qt < 0 ? NULL : a[3] != Py_None ? a[3] : a[2],
                                     kt < 0 ? NULL : a[5] != Py_None ? a[5] : a[4]))
    return NULL;
  return PyLong_FromLong(status);
}

/* ---- decode: pool, page_table, context_lens, q, scale, out, workspace, splits, stream;
 *      with weights_in and weights_out after the output ---- */
static PyObject* decode_call(int weigh, PyObject* const* a, Py_ssize_t na) {
  jf_kv_pool p;
  void *pt, *ctx, *q, *out, *ws, *stream, *w_in = NULL, *w_out = NULL;
  int64_t sh[4], qs[4], os[4], wi[4], wo[4] = {0, 0, 0, 0};
  if (want(weigh ? 11 : 9, na) || pool_of(a[0], &p) ||
      tensor(a[1], G.i32, "page_table", 1, I32_T, &pt) ||
      tensor(a[2], G.i32, "context_lens", 1, I32_T, &ctx) || tensor(a[3], G.bf16, "q", 1, BF16_T, &q) ||
      tensor(a[5], G.bf16, "out", 1, BF16_T, &out))
    return NULL;
  PyObject* const* r = a + 6;
  if (weigh) {
    if (tensor(a[7], G.f32, "weights_out", 1, F32_T, &w_out)) return NULL;
    r = a + 8;
  }
  if (tensor(r[0], G.u8, "workspace", 1, U8_T, &ws)) return NULL;
  const int nt = ints_of(a[1], 0, sh), nq = ints_of(a[3], 0, qs), no = ints_of(a[5], 0, os);
  if (nt < 0 || nq < 0 || no < 0) return NULL;
  if ((nt != 2 || nq != 3 || no != 3 || qs[0] != os[0] || qs[1] != os[1] || qs[2] != os[2] ||
       qs[2] != p.head_dim || sh[0] != qs[0] || numel(a[2]) != qs[0]) &&
      bad("shape mismatch"))
    return NULL;
  if (weigh) {
    const int n = ints_of(a[7], 0, wo);
    if (n < 0) return NULL;
    if ((n != 3 || wo[0] != qs[0] || wo[1] != p.num_kv_heads) &&
        bad("weights must be [batch, Hkv, stride]"))
      return NULL;
    if (a[6] != Py_None) {
      if (tensor(a[6], G.f32, "weights_in", 1, F32_T, &w_in)) return NULL;
      const int ni = ints_of(a[6], 0, wi);
      if (ni < 0) return NULL;
      if ((ni != 3 || wi[0] != wo[0] || wi[1] != wo[1] || wi[2] != wo[2]) &&
          bad("weights_in and weights_out must have one shape"))
        return NULL;
    }
  }
  const double scale = PyFloat_AsDouble(a[4]);
  int32_t splits;
  if (PyErr_Occurred() || int_of(r[1], &splits)) return NULL;
  const int64_t bytes = numel(r[0]);
  if (stream_of(r[2], &stream)) return NULL;
  if (fit(sh[1]) || fit(qs[0]) || fit(qs[1])) return NULL;
  if (weigh)
    CALL(G.weights(&p, pt, (int32_t)sh[1], ctx, (int32_t)qs[0], q, (int32_t)qs[1], (float)scale,
                   out, w_in, w_out, wo[2], ws, (size_t)bytes, splits, stream));
  CALL(G.decode(&p, pt, (int32_t)sh[1], ctx, (int32_t)qs[0], q, (int32_t)qs[1], (float)scale, out,
                ws, (size_t)bytes, splits, stream));
}
static PyObject* decode(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  (void)m;
  return decode_call(0, a, n);
}
static PyObject* decode_weights(PyObject* m, PyObject* const* a, Py_ssize_t n) {
  (void)m;
  return decode_call(1, a, n);
}

/* ---- evict: pool, page_table, context_lens, weights, budget, sinks, recent, dst_page_table,
 *      dst_context_lens, dst_weights, kept, err, stream ---- */
static PyObject* kv8_evict(PyObject* m, PyObject* const* a, Py_ssize_t na) {
  (void)m;
  jf_kv_pool p;
  void *pt, *ctx, *w, *dpt, *dctx, *dw = NULL, *kept, *err = NULL, *stream;
  int64_t sh[4], ws[4], ds[4], ks[4], dws[4];
  if (want(13, na) || pool_of(a[0], &p) || tensor(a[1], G.i32, "page_table", 1, I32_T, &pt) ||
      tensor(a[2], G.i32, "context_lens", 1, I32_T, &ctx) ||
      tensor(a[3], G.f32, "weights", 1, F32_T, &w) ||
      tensor(a[7], G.i32, "dst_page_table", 1, I32_T, &dpt) ||
      tensor(a[8], G.i32, "dst_context_lens", 1, I32_T, &dctx) ||
      tensor(a[10], G.i32, "kept", 1, I32_T, &kept) ||
      (a[9] != Py_None && tensor(a[9], G.f32, "dst_weights", 1, F32_T, &dw)) ||
      (a[11] != Py_None && tensor(a[11], G.i32, "err_flag", 1, I32_T, &err)))
    return NULL;
  int32_t budget, sinks, recent;
  if (int_of(a[4], &budget) || int_of(a[5], &sinks) || int_of(a[6], &recent)) return NULL;
  const int nt = ints_of(a[1], 0, sh), nw = ints_of(a[3], 0, ws), nd = ints_of(a[7], 0, ds),
            nk = ints_of(a[10], 0, ks);
  if (nt < 0 || nw < 0 || nd < 0 || nk < 0) return NULL;
  if ((nt != 2 || nd != 2 || ds[0] != sh[0] || numel(a[2]) != sh[0] || numel(a[8]) != sh[0]) &&
      bad("one row per request"))
    return NULL;
  if ((nw != 3 || ws[0] != sh[0] || ws[1] != p.num_kv_heads) && bad("weights must be [batch, Hkv, stride]"))
    return NULL;
  if ((nk != 3 || ks[0] != sh[0] || ks[1] != p.num_kv_heads || ks[2] != budget) &&
      bad("kept must be [batch, Hkv, budget]"))
    return NULL;
  if (dw) {
    const int n = ints_of(a[9], 0, dws);
    if (n < 0) return NULL;
    if ((n != 3 || dws[0] != ks[0] || dws[1] != ks[1] || dws[2] != ks[2]) &&
        bad("dst_weights must be [batch, Hkv, budget]"))
      return NULL;
  }
  if (stream_of(a[12], &stream)) return NULL;
  if (fit(sh[0]) || fit(sh[1]) || fit(ds[1])) return NULL;
  CALL(G.evict(&p, pt, (int32_t)sh[1], ctx, (int32_t)sh[0], w, ws[2], budget, sinks, recent, dpt,
               (int32_t)ds[1], dctx, dw, kept, err, stream));
}

/* ---- set-up: the entry points' addresses, torch's dtypes, stream and autograd functions ---- */
static PyObject* setup(PyObject* m, PyObject* args) {
  (void)m;
  unsigned long long f[6];
  PyObject *dt[5], *raw, *dev, *cur, *grad, *written;
  if (!PyArg_ParseTuple(args, "(KKKKKK)(OOOOO)OOOOO", f, f + 1, f + 2, f + 3, f + 4, f + 5, dt,
                        dt + 1, dt + 2, dt + 3, dt + 4, &raw, &dev, &cur, &grad, &written))
    return NULL;
  G.append = (rows_fn)(uintptr_t)f[0];
  G.read = (rows_fn)(uintptr_t)f[1];
  G.rope = (void*)(uintptr_t)f[2];
  G.decode = (void*)(uintptr_t)f[3];
  G.weights = (void*)(uintptr_t)f[4];
  G.evict = (void*)(uintptr_t)f[5];
  G.i32 = Py_NewRef(dt[0]);
  G.u8 = Py_NewRef(dt[1]);
  G.f32 = Py_NewRef(dt[2]);
  G.bf16 = Py_NewRef(dt[3]);
  G.f16 = Py_NewRef(dt[4]);
  G.raw_stream = raw == Py_None ? NULL : Py_NewRef(raw);
  G.get_device = Py_NewRef(dev);
  G.current_stream = Py_NewRef(cur);
  G.grad_enabled = Py_NewRef(grad);
  G.written = Py_NewRef(written);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {FAST(kv8_append), FAST(kv8_read), FAST(rope_axes), FAST(decode),
                                FAST(decode_weights), FAST(kv8_evict),
                                {"setup", setup, METH_VARARGS, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_jfcall", NULL, -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__jfcall(void) {
  const struct {
    PyObject** to;
    const char* text;
  } names[] = {{&s_dtype, "dtype"}, {&s_is_cuda, "is_cuda"}, {&s_contig, "is_contiguous"},
               {&s_ptr, "data_ptr"}, {&s_shape, "shape"}, {&s_stride, "stride"},
               {&s_numel, "numel"}, {&s_stream, "cuda_stream"},
               {&s_grad, "requires_grad"}, {&s_data, "data"},
               {&s_page, "page_size"}, {&s_hkv, "num_kv_heads"}, {&s_dim, "head_dim"},
               {&s_group, "group_size"}, {&s_format, "format"}};
  for (size_t i = 0; i < sizeof names / sizeof names[0]; ++i) {
    *names[i].to = PyUnicode_InternFromString(names[i].text);
    if (!*names[i].to) return NULL;
  }
  return PyModule_Create(&module);
}
