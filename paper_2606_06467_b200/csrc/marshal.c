/*
 * Argument marshalling of the 8-bit cache calls and of the calls around a layer for CPython: the checks and conversions of cache8.py
 * and layer.py without the interpreter. A decode step's operators run for 2 to 6 microseconds, and a call through ctypes spends as long on looking at its
 * tensors (16 tokens' clsa_norm_rope, called in a row: 7.95 us through ctypes, 5.4 through this module; the launch itself 3.9).
 *
 * Every function returns the call's clsa_status as an int, or None where its arguments are not exactly what it expects (a
 * device address in place of a tensor, another dtype, layout or device): the caller then takes the Python module's own path, which
 * accepts what is acceptable and words the errors. No state is kept between calls.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "clsa_layer.h"

typedef clsa_status (*norm_rope_fn)(const clsa_norm_rope_spec*, int32_t, const int32_t*, const clsa_heads*, const clsa_heads*,
                                    const clsa_heads*, const clsa_heads*, clsa_stream);
typedef clsa_status (*append_fn)(const clsa_params*, const clsa_cache8*, const clsa_norm_rope_spec*, const clsa_heads*, const clsa_heads*,
                                 const clsa_heads*, void*, size_t, clsa_stream);
typedef clsa_status (*scores_fn)(const clsa_params*, const clsa_cache8*, const void*, float*, int64_t, void*, size_t, clsa_stream);
typedef clsa_status (*attn_fn)(const clsa_params*, const clsa_cache8*, const void*, const int32_t*, const int32_t*, void*, float*,
                               const clsa_attn_hints*, void*, size_t, clsa_stream);

typedef clsa_status (*dense_fn)(const clsa_params*, int32_t, const void*, void*, float*, void*, size_t, clsa_stream);
typedef clsa_status (*dense8_fn)(const clsa_params*, const clsa_cache8*, int32_t, const void*, void*, float*, void*, size_t, clsa_stream);
typedef clsa_status (*add_norm_fn)(const clsa_add_norm_spec*, int32_t, const clsa_rows*, const clsa_rows*, const clsa_rows*, const clsa_rows*,
                                   const clsa_rows*, const clsa_rows*, clsa_stream);
typedef clsa_status (*axes_fn)(const clsa_norm_rope_spec*, const clsa_rope_axes*, int32_t, const int32_t*, int64_t, const clsa_heads*,
                               const clsa_heads*, const clsa_heads*, const clsa_heads*, clsa_stream);

static norm_rope_fn f_norm_rope;
static append_fn f_append;
static scores_fn f_scores;
static attn_fn f_attn;
static dense_fn f_dense;
static dense8_fn f_dense8;
static add_norm_fn f_add_norm;
static axes_fn f_axes;
static PyObject *t_tensor, *t_bf16, *t_i32, *t_f32, *t_u8, *g_device, *g_stream;  /* torch's: type, dtypes, two functions */
static PyObject *t_params, *t_cache, *t_spec, *t_hints, *t_norm, *t_axes; /* the bindings' structs */
static PyObject *t_e4m3, *t_e8m0; /* torch's 8-bit dtypes */
static PyObject *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_get_device, *s_is_contiguous, *s_numel, *s__device, *s__extent, *s__made, *s__kv, *s__pairs, *s_cuda_stream;

/* What a call needs of a tensor. */
typedef struct {
  void* data;
  int nd;
  int64_t shape[4], stride[4];
} view;

static PyObject* ask(PyObject* t, PyObject* method) {
  PyObject* args[1] = {t};
  return PyObject_VectorcallMethod(method, args, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL);
}
/* An int that a method of t returns; -2 and *bad = 1 if there is none. */
static int64_t ask_int(PyObject* t, PyObject* method, int* bad) {
  PyObject* r = ask(t, method);
  if (r == NULL) { PyErr_Clear(); *bad = 1; return -2; }
  const int64_t v = PyLong_Check(r) ? PyLong_AsLongLong(r) : (*bad = 1, -2);
  Py_DECREF(r);
  if (PyErr_Occurred()) { PyErr_Clear(); *bad = 1; }
  return v;
}
static int is_tensor(PyObject* t, PyObject* dtype, int64_t device) {
  if ((PyObject*)Py_TYPE(t) != t_tensor) return 0;
  int bad = 0;
  if (dtype != NULL) {
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    if (d == NULL) { PyErr_Clear(); return 0; }
    bad = d != dtype;
    Py_DECREF(d);
    if (bad) return 0;
  }
  return ask_int(t, s_get_device, &bad) == device && !bad;
}
static void* data_of(PyObject* t, int* bad) { return (void*)(uintptr_t)ask_int(t, s_data_ptr, bad); }
static int sizes(PyObject* tuple, int64_t* out) { /* up to four ints; their number, or -1 */
  if (tuple == NULL) { PyErr_Clear(); return -1; }
  int n = -1;
  if (PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) <= 4) {
    n = (int)PyTuple_GET_SIZE(tuple);
    for (int i = 0; i < n; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
    if (PyErr_Occurred()) { PyErr_Clear(); n = -1; }
  }
  Py_DECREF(tuple);
  return n;
}
static int look(PyObject* t, PyObject* dtype, int64_t device, view* v) {
  if (!is_tensor(t, dtype, device)) return 0;
  int bad = 0;
  v->nd = sizes(PyObject_GetAttr(t, s_shape), v->shape);
  if (v->nd < 1 || sizes(ask(t, s_stride), v->stride) != v->nd) return 0;
  v->data = data_of(t, &bad);
  return !bad;
}
/* The address of a dense tensor of `need` elements or more; 0 if it is not one. None gives NULL where it is allowed. */
static int dense(PyObject* t, PyObject* dtype, int64_t device, int none_ok, double need, void** out) {
  *out = NULL;
  if (t == Py_None) return none_ok;
  if (!is_tensor(t, dtype, device)) return 0;
  PyObject* c = ask(t, s_is_contiguous);
  if (c == NULL) { PyErr_Clear(); return 0; }
  int bad = c != Py_True;
  Py_DECREF(c);
  if (bad || (double)ask_int(t, s_numel, &bad) < need || bad) return 0;
  *out = data_of(t, &bad);
  return !bad;
}
/* Heads of [tokens, heads, dim] or [B, T, heads, dim] ([.., dim] with flat: one head). */
static int heads_of(PyObject* t, int64_t device, int64_t dim, int flat, clsa_heads* h, int64_t* tokens) {
  view v;
  if (!look(t, t_bf16, device, &v)) return 0;
  if (flat) {
    if (v.nd > 3) return 0;
    v.shape[v.nd] = v.shape[v.nd - 1];
    v.stride[v.nd] = v.stride[v.nd - 1];
    v.shape[v.nd - 1] = 1;
    v.stride[v.nd - 1] = dim;
    v.nd += 1;
  }
  int64_t token;
  if (v.nd == 3) {
    *tokens = v.shape[0];
    token = v.stride[0];
  } else if (v.nd == 4) {
    *tokens = v.shape[0] * v.shape[1];
    if (v.shape[1] != 1 && v.shape[0] != 1 && *tokens != 0 && v.stride[0] != v.shape[1] * v.stride[1]) return 0;
    token = v.shape[1] == 1 ? v.stride[0] : v.stride[1];
  } else {
    return 0;
  }
  const int64_t n = v.shape[v.nd - 2];
  if (v.shape[v.nd - 1] != dim || v.stride[v.nd - 1] != 1 || n > 0x7fffffff) return 0;
  h->data = v.data;
  h->num_heads = (int32_t)n;
  h->token_stride = token;
  h->head_stride = n > 1 ? v.stride[v.nd - 2] : dim;
  return 1;
}
/* A ctypes struct's bytes (which stay where they are while the caller holds it), if its tensors are on the device. */
static const void* struct_of(PyObject* s, PyObject* type, Py_ssize_t bytes, int64_t device, int tensors) {
  if ((PyObject*)Py_TYPE(s) != type) return NULL;
  if (tensors) {
    PyObject* d = PyObject_GetAttr(s, s__device);
    if (d == NULL) { PyErr_Clear(); return NULL; }
    const int ok = d == Py_None || (PyLong_Check(d) && PyLong_AsLongLong(d) == device);
    Py_DECREF(d);
    if (!ok) return NULL;
  }
  Py_buffer b;
  if (PyObject_GetBuffer(s, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return NULL; }
  const void* p = b.len == bytes ? b.buf : NULL;
  PyBuffer_Release(&b);
  return p;
}
/* Whether a cache's tensors, if it was made of tensors, hold what the params name of K and V, and of K_idx. */
static int fits(PyObject* cache, const clsa_cache8* c, const clsa_params* p, int kv, int idx) {
  int64_t e[7]; /* rows, heads, dimension; rows and dimension of K_idx; addresses of K and K_idx */
  PyObject* t = PyObject_GetAttr(cache, s__extent);
  if (t == NULL) { PyErr_Clear(); return 0; }
  int ok = t == Py_None;
  if (!ok && PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 7) {
    for (int i = 0; i < 7; ++i) e[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    kv = kv && (int64_t)(uintptr_t)c->k == e[5];
    idx = idx && (int64_t)(uintptr_t)c->idx_k == e[6];
    ok = !PyErr_Occurred() && !(kv && e[1] > 0 && (p->num_cache_rows > e[0] || p->num_kv_heads > e[1] || p->head_dim > e[2])) &&
         !(idx && e[4] > 0 && (p->num_cache_rows > e[3] || p->idx_dim > e[4]));
    PyErr_Clear();
  }
  Py_DECREF(t);
  return ok;
}
/* Whether the tensors that the params were made of describe all their sequences and lie on the device. */
static int describes(PyObject* params, const clsa_params* p, int64_t device) {
  const void* now[3] = {p->block_table == NULL ? p->seq_start : NULL, p->seq_len, p->block_table};
  PyObject* t = PyObject_GetAttr(params, s__made);
  if (t == NULL) { PyErr_Clear(); return 0; }
  int ok = t == Py_None || (PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 3);
  for (int i = 0; i < 3 && ok && t != Py_None; ++i) {
    PyObject* m = PyTuple_GET_ITEM(t, i); /* address, sequences, device or None */
    if (m == Py_None) continue;
    ok = PyTuple_Check(m) && PyTuple_GET_SIZE(m) == 3;
    if (!ok || now[i] == NULL || PyLong_AsLongLong(PyTuple_GET_ITEM(m, 0)) != (int64_t)(uintptr_t)now[i]) continue;
    PyObject* d = PyTuple_GET_ITEM(m, 2);
    ok = PyLong_AsLongLong(PyTuple_GET_ITEM(m, 1)) >= p->num_seqs && (d == Py_None || PyLong_AsLongLong(d) == device);
  }
  if (PyErr_Occurred()) { PyErr_Clear(); ok = 0; }
  Py_DECREF(t);
  return ok;
}
/* The current device, -1 if there is none. */
static int64_t current_device(void) {
  PyObject* r = PyObject_CallNoArgs(g_device);
  if (r == NULL) { PyErr_Clear(); return -1; }
  const int64_t v = PyLong_Check(r) ? PyLong_AsLongLong(r) : -1;
  Py_DECREF(r);
  if (PyErr_Occurred()) { PyErr_Clear(); return -1; }
  return v;
}
static int stream_of(PyObject* stream, int64_t device, clsa_stream* out) {
  PyObject* r = NULL;
  if (stream == Py_None) {
    PyObject* d = PyLong_FromLongLong(device);
    if (d == NULL) { PyErr_Clear(); return 0; }
    r = PyObject_CallOneArg(g_stream, d);
    Py_DECREF(d);
  } else if (PyLong_Check(stream)) {
    r = Py_NewRef(stream);
  } else {
    r = PyObject_GetAttr(stream, s_cuda_stream);
  }
  if (r == NULL) { PyErr_Clear(); return 0; }
  const int ok = PyLong_Check(r);
  *out = ok ? (clsa_stream)(uintptr_t)PyLong_AsUnsignedLongLong(r) : NULL;
  Py_DECREF(r);
  if (PyErr_Occurred()) { PyErr_Clear(); return 0; }
  return ok;
}
static int workspace_of(PyObject* ws, PyObject* bytes, int64_t device, void** out, size_t* n) {
  int bad = 0;
  if (!is_tensor(ws, t_u8, device)) return 0;
  const size_t has = (size_t)ask_int(ws, s_numel, &bad);
  if (bytes == Py_None) *n = has;
  else if (PyLong_Check(bytes)) *n = (size_t)PyLong_AsUnsignedLongLong(bytes);
  else return 0;
  if (PyErr_Occurred()) { PyErr_Clear(); return 0; }
  if (*n > has) return 0;
  *out = data_of(ws, &bad);
  return !bad;
}

/* Whether the tensors that K and V were made of are bf16, on the device and large enough. */
static int holds(PyObject* params, const clsa_params* p, int64_t device) {
  const void* now[2] = {p->k_cache, p->v_cache};
  const int64_t need = (p->num_cache_rows - 1) * p->kv_token_stride + (p->num_kv_heads - 1) * p->kv_head_stride + p->head_dim;
  PyObject* t = PyObject_GetAttr(params, s__kv);
  if (t == NULL) { PyErr_Clear(); return 0; }
  int ok = t == Py_None || (PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 2);
  for (int i = 0; i < 2 && ok && t != Py_None; ++i) {
    PyObject* m = PyTuple_GET_ITEM(t, i); /* address, dtype, elements, device */
    if (m == Py_None) continue;
    ok = PyTuple_Check(m) && PyTuple_GET_SIZE(m) == 4;
    if (!ok || PyLong_AsLongLong(PyTuple_GET_ITEM(m, 0)) != (int64_t)(uintptr_t)now[i]) continue;
    PyObject* d = PyTuple_GET_ITEM(m, 1);
    ok = PyUnicode_Check(d) && PyUnicode_CompareWithASCIIString(d, "torch.bfloat16") == 0 && PyLong_AsLongLong(PyTuple_GET_ITEM(m, 2)) >= need &&
         PyLong_AsLongLong(PyTuple_GET_ITEM(m, 3)) == device;
  }
  if (PyErr_Occurred()) { PyErr_Clear(); ok = 0; }
  Py_DECREF(t);
  return ok;
}
/* A matrix [.., length] whose rows are evenly spaced, of one of two dtypes; *rows: its rows, or (>= 0) what they have to be. */
static int matrix_of(PyObject* t, PyObject* dtype, PyObject* other, int64_t device, int64_t length, int64_t* rows, clsa_rows* out) {
  view v;
  if (!look(t, dtype, device, &v) && (other == NULL || !look(t, other, device, &v))) return 0;
  if (v.shape[v.nd - 1] != length || (v.stride[v.nd - 1] != 1 && length != 1)) return 0;
  int64_t n = 1, step = -1;
  int none = 0; /* no rows at all: nothing is spaced */
  for (int i = v.nd - 2; i >= 0; --i) none |= v.shape[i] == 0;
  for (int i = v.nd - 2; i >= 0; --i) {
    if (v.shape[i] == 1) continue;
    if (step < 0) step = v.stride[i];
    else if (v.stride[i] != n * step && !none) return 0;
    n *= v.shape[i];
  }
  if ((*rows >= 0 && n != *rows) || n > 0x7fffffff) return 0;
  *rows = n;
  out->data = v.data;
  out->stride = step < 0 ? length : step;
  return 1;
}

#define FALL_BACK Py_RETURN_NONE
#define RUN(call)                   \
  clsa_status st;                   \
  Py_BEGIN_ALLOW_THREADS st = call; \
  Py_END_ALLOW_THREADS return PyLong_FromLong((long)st)

/* spec, positions, q, q_out, k, k_out, stream */
static PyObject* m_norm_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  if (n != 7 || f_norm_rope == NULL || (a[2] == Py_None && a[4] == Py_None)) FALL_BACK;
  const int64_t dev = current_device();
  const clsa_norm_rope_spec* spec = (const clsa_norm_rope_spec*)struct_of(a[0], t_spec, sizeof(*spec), dev, 1);
  if (dev < 0 || spec == NULL) FALL_BACK;
  clsa_heads h[4];
  const clsa_heads* p[4] = {NULL, NULL, NULL, NULL};
  int64_t tokens = -1;
  for (int i = 0; i < 4; ++i) {
    if (a[2 + i] == Py_None) {
      if (a[2 + (i ^ 1)] != Py_None) FALL_BACK;
      continue;
    }
    int64_t t;
    if (!heads_of(a[2 + i], dev, spec->head_dim, 0, &h[i], &t) || (tokens >= 0 && t != tokens)) FALL_BACK;
    if ((i & 1) && h[i].num_heads != h[i - 1].num_heads) FALL_BACK;
    tokens = t;
    p[i] = &h[i];
  }
  void* pos;
  if (!dense(a[1], t_i32, dev, 1, (double)tokens, &pos) || tokens > 0x7fffffff) FALL_BACK;
  if (pos != NULL) {
    int bad = 0;
    if (ask_int(a[1], s_numel, &bad) != tokens || bad) FALL_BACK;
  }
  clsa_stream s;
  if (!stream_of(a[6], dev, &s)) FALL_BACK;
  RUN(f_norm_rope(spec, (int32_t)tokens, (const int32_t*)pos, p[0], p[1], p[2], p[3], s));
}

/* p, c, spec, k_new, v_new, idx_k_new, workspace, workspace_bytes, stream */
static PyObject* m_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  if (n != 9 || f_append == NULL || (a[3] == Py_None) != (a[4] == Py_None) || (a[3] == Py_None && a[5] == Py_None)) FALL_BACK;
  const int64_t dev = current_device();
  const clsa_params* p = (const clsa_params*)struct_of(a[0], t_params, sizeof(*p), dev, 0);
  const clsa_cache8* c = (const clsa_cache8*)struct_of(a[1], t_cache, sizeof(*c), dev, 1);
  const clsa_norm_rope_spec* spec = a[2] == Py_None ? NULL : (const clsa_norm_rope_spec*)struct_of(a[2], t_spec, sizeof(*spec), dev, 1);
  if (dev < 0 || p == NULL || c == NULL || (a[2] != Py_None && spec == NULL) || !describes(a[0], p, dev) || !fits(a[1], c, p, a[3] != Py_None, a[5] != Py_None)) FALL_BACK;
  clsa_heads h[3];
  const clsa_heads* q[3] = {NULL, NULL, NULL};
  for (int i = 0; i < 3; ++i) {
    if (a[3 + i] == Py_None) continue;
    int64_t t;
    if (!heads_of(a[3 + i], dev, i < 2 ? p->head_dim : p->idx_dim, i == 2, &h[i], &t)) FALL_BACK;
    if (t != (int64_t)p->num_seqs * p->q_per_seq || h[i].num_heads != (i < 2 ? p->num_kv_heads : 1)) FALL_BACK;
    q[i] = &h[i];
  }
  void* ws;
  size_t bytes;
  clsa_stream s;
  if (!workspace_of(a[6], a[7], dev, &ws, &bytes) || !stream_of(a[8], dev, &s)) FALL_BACK;
  RUN(f_append(p, c, spec, q[0], q[1], q[2], ws, bytes, s));
}

/* p, c, q_idx, scores, score_stride, workspace, workspace_bytes, stream */
static PyObject* m_scores(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  if (n != 8 || f_scores == NULL || !PyLong_Check(a[4])) FALL_BACK;
  const int64_t dev = current_device();
  const clsa_params* p = (const clsa_params*)struct_of(a[0], t_params, sizeof(*p), dev, 0);
  const clsa_cache8* c = (const clsa_cache8*)struct_of(a[1], t_cache, sizeof(*c), dev, 1);
  void *q, *sc, *ws;
  size_t bytes;
  clsa_stream s;
  const int64_t stride = PyLong_AsLongLong(a[4]);
  if (PyErr_Occurred()) { PyErr_Clear(); FALL_BACK; }
  if (dev < 0 || p == NULL || c == NULL || !describes(a[0], p, dev) || !fits(a[1], c, p, 0, 1)) FALL_BACK;
  const double rows = (double)p->num_seqs * p->q_per_seq;
  if (!dense(a[2], t_bf16, dev, 0, rows * p->idx_dim, &q) || !dense(a[3], t_f32, dev, 0, (rows - 1) * (double)stride + p->max_seq_len, &sc) ||
      !workspace_of(a[5], a[6], dev, &ws, &bytes) || !stream_of(a[7], dev, &s))
    FALL_BACK;
  RUN(f_scores(p, c, q, (float*)sc, stride, ws, bytes, s));
}

/* p, c, q, idx, count, out, lse, hints, workspace, workspace_bytes, stream */
static PyObject* m_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  if (n != 11 || f_attn == NULL) FALL_BACK;
  const int64_t dev = current_device();
  const clsa_params* p = (const clsa_params*)struct_of(a[0], t_params, sizeof(*p), dev, 0);
  const clsa_cache8* c = (const clsa_cache8*)struct_of(a[1], t_cache, sizeof(*c), dev, 1);
  const clsa_attn_hints* hints = a[7] == Py_None ? NULL : (const clsa_attn_hints*)struct_of(a[7], t_hints, sizeof(*hints), dev, 0);
  void *q, *idx, *count, *out, *lse, *ws;
  size_t bytes;
  clsa_stream s;
  if (dev < 0 || p == NULL || c == NULL || (a[7] != Py_None && hints == NULL) || !describes(a[0], p, dev) || !fits(a[1], c, p, 1, 0)) FALL_BACK;
  const double rows = (double)p->num_seqs * p->q_per_seq, heads = rows * p->num_q_heads;
  if (!dense(a[2], t_bf16, dev, 0, heads * p->head_dim, &q) || !dense(a[3], t_i32, dev, 0, rows * p->top_k, &idx) ||
      !dense(a[4], t_i32, dev, 0, rows, &count) || !dense(a[5], t_bf16, dev, 0, heads * p->head_dim, &out) ||
      !dense(a[6], t_f32, dev, 1, heads, &lse) || !workspace_of(a[8], a[9], dev, &ws, &bytes) || !stream_of(a[10], dev, &s))
    FALL_BACK;
  RUN(f_attn(p, c, q, (const int32_t*)idx, (const int32_t*)count, out, (float*)lse, hints, ws, bytes, s));
}

/* p, window, q, out, lse, workspace, workspace_bytes, stream; with an 8-bit cache behind p */
static PyObject* dense_call(PyObject* const* a, Py_ssize_t n, int eight) {
  if (n != 8 + eight || f_dense == NULL) FALL_BACK;
  PyObject *params = a[0], *cache = eight ? a[1] : NULL;
  a += eight;
  const int64_t dev = current_device();
  const clsa_params* p = (const clsa_params*)struct_of(params, t_params, sizeof(*p), dev, 0);
  const clsa_cache8* c = eight ? (const clsa_cache8*)struct_of(cache, t_cache, sizeof(*c), dev, 1) : NULL;
  if (dev < 0 || p == NULL || (eight && c == NULL) || !PyLong_Check(a[1]) || !describes(params, p, dev)) FALL_BACK;
  if (eight ? !fits(cache, c, p, 1, 0) : !holds(params, p, dev)) FALL_BACK;
  const long long window = PyLong_AsLongLong(a[1]);
  if (PyErr_Occurred()) { PyErr_Clear(); FALL_BACK; }
  if (window < 0 || window > 0x7fffffff) FALL_BACK;
  const double heads = (double)p->num_seqs * p->q_per_seq * p->num_q_heads;
  void *q, *out, *lse, *ws;
  size_t bytes;
  clsa_stream s;
  if (!dense(a[2], t_bf16, dev, 0, heads * p->head_dim, &q) || !dense(a[3], t_bf16, dev, 0, heads * p->head_dim, &out) ||
      !dense(a[4], t_f32, dev, 1, heads, &lse) || !workspace_of(a[5], a[6], dev, &ws, &bytes) || !stream_of(a[7], dev, &s))
    FALL_BACK;
  if (eight) { RUN(f_dense8(p, c, (int32_t)window, q, out, (float*)lse, ws, bytes, s)); }
  RUN(f_dense(p, (int32_t)window, q, out, (float*)lse, ws, bytes, s));
}
static PyObject* m_dense(PyObject* self, PyObject* const* a, Py_ssize_t n) { (void)self; return dense_call(a, n, 0); }
static PyObject* m_dense8(PyObject* self, PyObject* const* a, Py_ssize_t n) { (void)self; return dense_call(a, n, 1); }

/* spec, x, residual, sum_out, y_out, codes_out, scales_out, stream */
static PyObject* m_add_norm(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  if (n != 8 || f_add_norm == NULL || (a[5] == Py_None) != (a[6] == Py_None) || (a[4] == Py_None && a[5] == Py_None)) FALL_BACK;
  const int64_t dev = current_device();
  const clsa_add_norm_spec* spec = (const clsa_add_norm_spec*)struct_of(a[0], t_norm, sizeof(*spec), dev, 1);
  if (dev < 0 || spec == NULL || (a[5] != Py_None && spec->scale_group < 1)) FALL_BACK;
  clsa_rows m[6];
  const clsa_rows* p[6] = {NULL, NULL, NULL, NULL, NULL, NULL};
  int64_t rows = -1;
  for (int i = 0; i < 6; ++i) {
    if (a[1 + i] == Py_None) {
      if (i == 0) FALL_BACK;
      continue;
    }
    PyObject *type = i < 4 ? t_bf16 : t_u8, *other = i == 4 ? t_e4m3 : i == 5 ? t_e8m0 : NULL;
    if (!matrix_of(a[1 + i], type, other, dev, i == 5 ? spec->dim / spec->scale_group : spec->dim, &rows, &m[i])) FALL_BACK;
    p[i] = &m[i];
  }
  clsa_stream s;
  if (!stream_of(a[7], dev, &s)) FALL_BACK;
  RUN(f_add_norm(spec, (int32_t)rows, p[0], p[1], p[2], p[3], p[4], p[5], s));
}

/* spec, axes, positions, q, q_out, k, k_out, stream */
static PyObject* m_norm_rope_axes(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  if (n != 8 || f_axes == NULL || (a[3] == Py_None && a[5] == Py_None)) FALL_BACK;
  const int64_t dev = current_device();
  const clsa_norm_rope_spec* spec = (const clsa_norm_rope_spec*)struct_of(a[0], t_spec, sizeof(*spec), dev, 1);
  const clsa_rope_axes* axes = (const clsa_rope_axes*)struct_of(a[1], t_axes, sizeof(*axes), dev, 0);
  if (dev < 0 || spec == NULL || axes == NULL) FALL_BACK;
  PyObject* pairs = PyObject_GetAttr(a[1], s__pairs);
  if (pairs == NULL) { PyErr_Clear(); FALL_BACK; }
  const int agree = pairs == Py_None || (PyLong_Check(pairs) && PyLong_AsLongLong(pairs) * 2 == spec->rot_dim);
  Py_DECREF(pairs);
  if (!agree) FALL_BACK;
  clsa_heads h[4];
  const clsa_heads* p[4] = {NULL, NULL, NULL, NULL};
  int64_t tokens = -1;
  for (int i = 0; i < 4; ++i) {
    if (a[3 + i] == Py_None) {
      if (a[3 + (i ^ 1)] != Py_None) FALL_BACK;
      continue;
    }
    int64_t t;
    if (!heads_of(a[3 + i], dev, spec->head_dim, 0, &h[i], &t) || (tokens >= 0 && t != tokens)) FALL_BACK;
    if ((i & 1) && h[i].num_heads != h[i - 1].num_heads) FALL_BACK;
    tokens = t;
    p[i] = &h[i];
  }
  view v;
  if (tokens > 0x7fffffff || !look(a[2], t_i32, dev, &v) || v.nd > 2 || v.shape[v.nd - 1] != tokens || (v.stride[v.nd - 1] != 1 && tokens > 1)) FALL_BACK;
  if (v.nd == 2 && (v.shape[0] != axes->num_axes || (v.stride[0] > 0 && v.stride[0] < tokens))) FALL_BACK;
  clsa_stream s;
  if (!stream_of(a[7], dev, &s)) FALL_BACK;
  RUN(f_axes(spec, axes, (int32_t)tokens, (const int32_t*)v.data, v.nd == 2 && axes->num_axes > 1 ? v.stride[0] : 0, p[0], p[1], p[2], p[3], s));
}

/* The addresses of clsa_norm_rope, clsa_cache8_append, clsa_index_scores8, clsa_sparse_attn8; torch.Tensor, torch.bfloat16, .int32,
 * .float32, .uint8; the functions that give the current device and its current stream; the structs' types. */
static PyObject* m_setup(PyObject* self, PyObject* args) {
  (void)self;
  unsigned long long f[4];
  PyObject* o[11];
  if (!PyArg_ParseTuple(args, "KKKKOOOOOOOOOOO", &f[0], &f[1], &f[2], &f[3], &o[0], &o[1], &o[2], &o[3], &o[4], &o[5], &o[6], &o[7], &o[8], &o[9], &o[10])) return NULL;
  PyObject** to[11] = {&t_tensor, &t_bf16, &t_i32, &t_f32, &t_u8, &g_device, &g_stream, &t_params, &t_cache, &t_spec, &t_hints};
  for (int i = 0; i < 11; ++i) Py_XSETREF(*to[i], Py_NewRef(o[i]));
  f_norm_rope = (norm_rope_fn)(uintptr_t)f[0];
  f_append = (append_fn)(uintptr_t)f[1];
  f_scores = (scores_fn)(uintptr_t)f[2];
  f_attn = (attn_fn)(uintptr_t)f[3];
  Py_RETURN_NONE;
}
/* The addresses of clsa_dense_attn, clsa_dense_attn8, clsa_add_norm, clsa_norm_rope_axes; torch.float8_e4m3fn and .float8_e8m0fnu; the
 * structs' types (behind setup). */
static PyObject* m_setup_layer(PyObject* self, PyObject* args) {
  (void)self;
  unsigned long long f[4];
  PyObject* o[4];
  if (!PyArg_ParseTuple(args, "KKKKOOOO", &f[0], &f[1], &f[2], &f[3], &o[0], &o[1], &o[2], &o[3])) return NULL;
  PyObject** to[4] = {&t_e4m3, &t_e8m0, &t_norm, &t_axes};
  for (int i = 0; i < 4; ++i) Py_XSETREF(*to[i], Py_NewRef(o[i]));
  f_dense = (dense_fn)(uintptr_t)f[0];
  f_dense8 = (dense8_fn)(uintptr_t)f[1];
  f_add_norm = (add_norm_fn)(uintptr_t)f[2];
  f_axes = (axes_fn)(uintptr_t)f[3];
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"setup", m_setup, METH_VARARGS, NULL},
                                {"setup_layer", m_setup_layer, METH_VARARGS, NULL},
                                {"dense", (PyCFunction)(void (*)(void))m_dense, METH_FASTCALL, NULL},
                                {"dense8", (PyCFunction)(void (*)(void))m_dense8, METH_FASTCALL, NULL},
                                {"add_norm", (PyCFunction)(void (*)(void))m_add_norm, METH_FASTCALL, NULL},
                                {"norm_rope_axes", (PyCFunction)(void (*)(void))m_norm_rope_axes, METH_FASTCALL, NULL},
                                {"norm_rope", (PyCFunction)(void (*)(void))m_norm_rope, METH_FASTCALL, NULL},
                                {"append", (PyCFunction)(void (*)(void))m_append, METH_FASTCALL, NULL},
                                {"scores", (PyCFunction)(void (*)(void))m_scores, METH_FASTCALL, NULL},
                                {"attn", (PyCFunction)(void (*)(void))m_attn, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  struct { PyObject** to; const char* name; } names[] = {
      {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_data_ptr, "data_ptr"}, {&s_get_device, "get_device"},
      {&s_is_contiguous, "is_contiguous"}, {&s_numel, "numel"}, {&s__device, "_device"}, {&s__extent, "_extent"}, {&s__made, "_made"}, {&s__kv, "_kv"}, {&s__pairs, "_pairs"}, {&s_cuda_stream, "cuda_stream"}};
  for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
    if ((*names[i].to = PyUnicode_InternFromString(names[i].name)) == NULL) return NULL;
  return PyModule_Create(&module);
}
