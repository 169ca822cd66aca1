/* Argument marshalling of the Python binding (module _binding): tensors, views and plain values of one call go straight
 * into the C ABI's argument structs.  A call used to fill them field by field through ctypes (9 us for
 * lightkv_compress_layer, 6 for lightkv_compact_kv, more than the launches behind them take); here a tensor costs a
 * data_ptr() and a stride() call.  Needs no header of torch: tensors are Python objects with those two methods. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "lightkv.h"

typedef int (*layer_fn)(const lightkv_plan_t*, const lightkv_layer_args_t*);
typedef int (*kv_fn)(const lightkv_plan_t*, const lightkv_kv_args_t*);
typedef int (*decode_fn)(const lightkv_decode_args_t*);
typedef int (*append_fn)(const lightkv_append_args_t*);
typedef int (*pages_fn)(const lightkv_pages_args_t*);
static layer_fn g_layer, g_layer_builtin;
static kv_fn g_kv;
static decode_fn g_decode;
static append_fn g_append;
static pages_fn g_pages;
static PyObject *g_fail, *g_fork_join, *g_raw_stream, *g_device;   /* Python callables, see bind() */
static PyObject *g_bf16, *g_fp32, *g_i32, *g_i64;                  /* torch's dtypes */

/* names used as keywords, attributes or methods, interned once */
#define NAMES(X) \
  X(plan) X(stage) X(hidden) X(out) X(vis_begin) X(n_text_after) X(text_begin) X(text_end) X(q) X(k) X(lse) X(xi) \
  X(n_vis) X(pos) X(stream) X(trace_events) X(aux_stream) X(map_event) X(fork_event) X(join_event) X(text_ranges) \
  X(bidirectional) X(lse_out) X(seq_start) X(seq_start_out) X(hidden_out) X(k_src) X(v_src) X(k_dst) X(v_dst) X(mode) \
  X(page_size) X(src_block_table) X(dst_block_table) X(src_seq_start) X(dst_seq_start) X(data_ptr) X(size) \
  X(handle) X(value) X(n_vis_out) X(pos_out) X(dst) X(weight) X(grp_off) X(grp_src) X(xi_out) X(status) X(workspace) \
  X(info) X(workspace_bytes) X(cuda_stream) X(cuda_event) X(k_cache) X(v_cache) X(n_keys) X(block_table) X(k_new) X(v_new) \
  X(scale) X(max_keys) X(slot_map) X(seq_len) X(free_pages) X(n_free) X(add) X(held) X(seq_len_out) X(n_free_out) \
  X(slot_start) X(slot_stride) X(dtype) X(shape) X(get_device) X(is_contiguous) X(nbytes)
enum {
#define X(n) N_##n,
  NAMES(X)
#undef X
  N_COUNT
};
static PyObject* g_name[N_COUNT];
static PyObject* g_stride;   /* "stride" */

/* value of keyword / positional argument `id`, NULL when absent or None */
typedef struct { PyObject* v[N_COUNT]; } Args;
static PyObject* get(const Args* a, int id) { return a->v[id] == Py_None ? NULL : a->v[id]; }

static int parse(Args* a, const char* fn, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames,
                 const int* positional, int n_pos, int n_required, const int* keywords, int n_kw, int needed) {
  memset(a, 0, sizeof(*a));
  if (nargs > n_pos) { PyErr_Format(PyExc_TypeError, "%s() takes %d positional arguments but %zd were given", fn, n_pos, nargs); return -1; }
  for (Py_ssize_t i = 0; i < nargs; ++i) a->v[positional[i]] = args[i];
  const Py_ssize_t n = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* name = PyTuple_GET_ITEM(kwnames, i);
    int id = -1;
    for (int pass = 0; pass < 2 && id < 0; ++pass) {          /* interned names are equal as pointers */
      for (int j = 0; j < n_kw + n_pos && id < 0; ++j) {
        const int c = j < n_kw ? keywords[j] : positional[j - n_kw];
        if (pass == 0 ? name == g_name[c] : PyUnicode_Compare(name, g_name[c]) == 0) id = c;
      }
    }
    if (id < 0) { PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", fn, name); return -1; }
    if (a->v[id]) { PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%U'", fn, name); return -1; }
    a->v[id] = args[nargs + i];
  }
  for (int j = 0; j < n_required; ++j)
    if (!a->v[positional[j]]) { PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%U'", fn, g_name[positional[j]]); return -1; }
  if (!a->v[needed]) { PyErr_Format(PyExc_TypeError, "%s() missing 1 required keyword-only argument: '%U'", fn, g_name[needed]); return -1; }
  return 0;
}

static int to_i64(PyObject* v, int64_t* r) {
  if (PyLong_CheckExact(v)) { *r = PyLong_AsLongLong(v); return *r == -1 && PyErr_Occurred() ? -1 : 0; }
  PyObject* i = PyNumber_Index(v);                            /* numpy integers and the like */
  if (!i) return -1;
  *r = PyLong_AsLongLong(i);
  Py_DECREF(i);
  return *r == -1 && PyErr_Occurred() ? -1 : 0;
}
static int int_arg(const Args* a, int id, int32_t fallback, int32_t* r) {
  PyObject* v = get(a, id);
  int64_t t = fallback;
  if (v && to_i64(v, &t)) return -1;
  if (t < INT32_MIN || t > INT32_MAX) { PyErr_Format(PyExc_OverflowError, "'%U' is out of range", g_name[id]); return -1; }
  *r = (int32_t)t;
  return 0;
}
/* integer attribute of an object as a pointer (stream and event handles, plan handles) */
static int ptr_attr(PyObject* o, int id, void** r) {
  PyObject* v = PyObject_GetAttr(o, g_name[id]);
  if (!v) return -1;
  *r = v == Py_None ? NULL : PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !*r && PyErr_Occurred() ? -1 : 0;
}
/* address of a tensor's data; NULL object: NULL */
static int data(PyObject* t, void* r) {
  void* p = NULL;
  if (t) {
    PyObject* v = PyObject_CallMethodNoArgs(t, g_name[N_data_ptr]);
    if (!v) return -1;
    p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (!p && PyErr_Occurred()) return -1;
  }
  memcpy(r, &p, sizeof(p));
  return 0;
}
static int data_attr(PyObject* o, int id, void* r) {
  PyObject* t = PyObject_GetAttr(o, g_name[id]);
  if (!t) return -1;
  const int rc = data(t == Py_None ? NULL : t, r);
  Py_DECREF(t);
  return rc;
}
/* the first n strides of a tensor */
static int strides(PyObject* t, int n, int64_t* r) {
  PyObject* v = PyObject_CallMethodNoArgs(t, g_stride);
  if (!v) return -1;
  int rc = PyTuple_Check(v) && PyTuple_GET_SIZE(v) >= n ? 0 : -1;
  if (rc) PyErr_Format(PyExc_IndexError, "a tensor of at least %d dimensions is expected", n);
  for (int i = 0; i < n && !rc; ++i) rc = to_i64(PyTuple_GET_ITEM(v, i), &r[i]);
  Py_DECREF(v);
  return rc;
}
static int size_of(PyObject* t, int dim, int32_t* r) {
  PyObject* d = PyLong_FromLong(dim);
  PyObject* v = d ? PyObject_CallMethodOneArg(t, g_name[N_size], d) : NULL;
  Py_XDECREF(d);
  if (!v) return -1;
  *r = (int32_t)PyLong_AsLong(v);
  Py_DECREF(v);
  return *r == -1 && PyErr_Occurred() ? -1 : 0;
}
static int stream_handle(PyObject* stream, void** r) {
  if (stream) return ptr_attr(stream, N_cuda_stream, r);
  PyObject* dev = PyObject_CallNoArgs(g_device);              /* the current stream of the current device */
  PyObject* v = dev ? PyObject_CallOneArg(g_raw_stream, dev) : NULL;
  Py_XDECREF(dev);
  if (!v) return -1;
  *r = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !*r && PyErr_Occurred() ? -1 : 0;
}
static int plan_handle(PyObject* plan, void** r) {
  PyObject* h = PyObject_GetAttr(plan, g_name[N_handle]);
  if (!h) return -1;
  int rc = 0;
  *r = NULL;
  if (h != Py_None) rc = ptr_attr(h, N_value, r);
  Py_DECREF(h);
  return rc;
}
static PyObject* done(int code, const char* what) {
  if (code == 0) Py_RETURN_NONE;
  return PyObject_CallFunction(g_fail, "is", code, what);     /* raises LightKVError */
}

static const int kLayerPos[] = {N_plan, N_stage, N_hidden, N_out};
static const int kLayerKw[] = {N_vis_begin, N_n_text_after, N_q, N_k, N_n_vis, N_pos, N_lse, N_xi, N_text_begin, N_text_end,
                               N_stream, N_aux_stream, N_map_event, N_fork_event, N_join_event, N_trace_events, N_text_ranges,
                               N_bidirectional, N_lse_out, N_seq_start, N_seq_start_out, N_hidden_out};

static PyObject* layer(const char* fn, layer_fn call, int builtin, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  Args in;
  if (parse(&in, fn, args, nargs, kwnames, kLayerPos, 4, 4, kLayerKw, sizeof(kLayerKw) / sizeof(int), N_vis_begin)) return NULL;
  lightkv_layer_args_t a;
  memset(&a, 0, sizeof(a));
  a.struct_size = sizeof(a);
  PyObject *out = in.v[N_out], *t;
  void* plan;
  int64_t s[3];
  int32_t ranges[2 * LIGHTKV_MAX_TEXT_RANGES];
  void* trace[LIGHTKV_TRACE_EVENTS];
  if (plan_handle(in.v[N_plan], &plan) || int_arg(&in, N_stage, 0, &a.stage) || int_arg(&in, N_vis_begin, 0, &a.vis_begin) ||
      int_arg(&in, N_n_text_after, 0, &a.n_text_after) || int_arg(&in, N_text_begin, 0, &a.text_begin) ||
      int_arg(&in, N_text_end, a.vis_begin, &a.text_end))
    return NULL;
  if (data(in.v[N_hidden], &a.hidden) || strides(in.v[N_hidden], 2, s)) return NULL;
  a.hidden_batch_stride = s[0]; a.hidden_row_stride = s[1];
  t = get(&in, N_hidden_out);
  if (!t) t = PyObject_GetAttr(out, g_name[N_hidden_out]); else Py_INCREF(t);
  if (!t) return NULL;
  int rc = data(t, &a.hidden_out) || strides(t, 2, s);
  Py_DECREF(t);
  if (rc) return NULL;
  a.hidden_out_batch_stride = s[0]; a.hidden_out_row_stride = s[1];
  if ((t = get(&in, N_q))) {
    if (data(t, &a.q) || strides(t, 3, s) || size_of(t, 2, &a.seq_rows)) return NULL;
    a.q_batch_stride = s[0]; a.q_head_stride = s[1]; a.q_row_stride = s[2];
  }
  if ((t = get(&in, N_k))) {
    if (data(t, &a.k) || strides(t, 3, s)) return NULL;
    a.k_batch_stride = s[0]; a.k_head_stride = s[1]; a.k_row_stride = s[2];
  }
  if ((t = get(&in, N_lse))) {
    if (data(t, &a.lse) || strides(t, 2, s)) return NULL;
    a.lse_batch_stride = s[0]; a.lse_head_stride = s[1];
  }
  if ((t = get(&in, N_lse_out))) {
    if (data(t, &a.lse_out) || strides(t, 2, s)) return NULL;
    a.lse_out_batch_stride = s[0]; a.lse_out_head_stride = s[1];
  }
  if (data(get(&in, N_xi), &a.xi) || data(get(&in, N_n_vis), &a.n_vis) || data(get(&in, N_pos), &a.pos) ||
      data_attr(out, N_n_vis_out, &a.n_vis_out) || data_attr(out, N_pos_out, &a.pos_out) || data_attr(out, N_dst, &a.dst) ||
      data_attr(out, N_weight, &a.weight) || data_attr(out, N_grp_off, &a.grp_off) || data_attr(out, N_grp_src, &a.grp_src) ||
      data_attr(out, N_xi_out, &a.xi_out) || data_attr(out, N_status, &a.status))
    return NULL;
  if (!builtin) {
    void* p;
    PyObject* info = PyObject_GetAttr(out, g_name[N_info]);
    PyObject* bytes = info ? PyObject_GetAttr(info, g_name[N_workspace_bytes]) : NULL;
    Py_XDECREF(info);
    if (!bytes) return NULL;
    a.workspace_bytes = PyLong_AsSize_t(bytes);
    Py_DECREF(bytes);
    if (PyErr_Occurred() || data_attr(out, N_workspace, &p)) return NULL;
    a.workspace = (void*)(((uintptr_t)p + 255) / 256 * 256);
  }
  if (stream_handle(get(&in, N_stream), &a.stream)) return NULL;
  if ((t = get(&in, N_aux_stream))) {
    PyObject *fork = get(&in, N_fork_event), *join = get(&in, N_join_event), *pair = NULL;
    if (ptr_attr(t, N_cuda_stream, &a.aux_stream)) return NULL;
    if (!fork || !join) {                                     /* a pair kept with the stage's buffers */
      pair = PyObject_CallOneArg(g_fork_join, out);
      if (!pair) return NULL;
      fork = PyTuple_GET_ITEM(pair, 0); join = PyTuple_GET_ITEM(pair, 1);
    }
    rc = ptr_attr(fork, N_cuda_event, &a.fork_event) || ptr_attr(join, N_cuda_event, &a.join_event);
    Py_XDECREF(pair);
    if (rc) return NULL;
  }
  if ((t = get(&in, N_text_ranges))) {                        /* [(begin, end), ...] */
    PyObject* seq = PySequence_Fast(t, "text_ranges is a sequence of (begin, end)");
    if (!seq) return NULL;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    a.n_text_ranges = (int32_t)n;                             /* too many: the library refuses the count */
    a.text_ranges = ranges;
    for (Py_ssize_t i = 0; i < n && i < LIGHTKV_MAX_TEXT_RANGES && !rc; ++i)
      for (int e = 0; e < 2 && !rc; ++e) {
        PyObject* v = PySequence_GetItem(PySequence_Fast_GET_ITEM(seq, i), e);
        int64_t x = 0;
        rc = !v || to_i64(v, &x);
        Py_XDECREF(v);
        ranges[2 * i + e] = (int32_t)x;
      }
    Py_DECREF(seq);
    if (rc) return NULL;
  }
  if ((t = get(&in, N_bidirectional))) {
    a.bidirectional = PyObject_IsTrue(t);
    if (a.bidirectional < 0) return NULL;
  }
  if ((t = get(&in, N_seq_start))) {
    /* packed batch: tensors of shape [1, rows, ...] hold the samples back to back; sample b starts at row seq_start[b],
     * so the batch strides are 0 and q / k span all rows */
    if (data(t, &a.seq_start) || data(get(&in, N_seq_start_out), &a.seq_start_out)) return NULL;
    a.hidden_batch_stride = a.q_batch_stride = a.k_batch_stride = a.lse_batch_stride = a.lse_out_batch_stride = 0;
    if (a.seq_start_out) a.hidden_out_batch_stride = 0;
  }
  if ((t = get(&in, N_map_event)) && ptr_attr(t, N_cuda_event, &a.map_event)) return NULL;
  if ((t = get(&in, N_trace_events))) {
    PyObject* seq = PySequence_Fast(t, "trace_events is a sequence of events");
    if (!seq) return NULL;
    if (PySequence_Fast_GET_SIZE(seq) != LIGHTKV_TRACE_EVENTS) {
      PyErr_Format(PyExc_AssertionError, "%d trace events are expected", LIGHTKV_TRACE_EVENTS);
      rc = -1;
    }
    for (int i = 0; i < LIGHTKV_TRACE_EVENTS && !rc; ++i) rc = ptr_attr(PySequence_Fast_GET_ITEM(seq, i), N_cuda_event, &trace[i]);
    Py_DECREF(seq);
    if (rc) return NULL;
    a.trace_events = trace;
  }
  Py_BEGIN_ALLOW_THREADS
  rc = call(plan, &a);
  Py_END_ALLOW_THREADS
  return done(rc, builtin ? "lightkv_compress_layer_builtin_ws" : "lightkv_compress_layer");
}

static PyObject* compress_layer(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  return layer("compress_layer", g_layer, 0, args, nargs, kwnames);
}
static PyObject* compress_layer_builtin_ws(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  return layer("compress_layer_builtin_ws", g_layer_builtin, 1, args, nargs, kwnames);
}

static const int kKvPos[] = {N_plan, N_stage, N_out, N_k_src, N_v_src, N_k_dst, N_v_dst, N_vis_begin, N_n_text_after, N_mode,
                             N_n_vis, N_page_size, N_src_block_table, N_dst_block_table, N_stream, N_src_seq_start,
                             N_dst_seq_start};

static PyObject* compact_kv(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  Args in;
  if (parse(&in, "compact_kv", args, nargs, kwnames, kKvPos, sizeof(kKvPos) / sizeof(int), 8, NULL, 0, N_vis_begin)) return NULL;
  lightkv_kv_args_t a;
  memset(&a, 0, sizeof(a));
  a.struct_size = sizeof(a);
  PyObject* out = in.v[N_out];
  void* plan;
  int64_t s[4][3];
  if (plan_handle(in.v[N_plan], &plan) || int_arg(&in, N_stage, 0, &a.stage) || int_arg(&in, N_vis_begin, 0, &a.vis_begin) ||
      int_arg(&in, N_n_text_after, 0, &a.n_text_after) || int_arg(&in, N_mode, LIGHTKV_KV_MERGE, &a.mode) ||
      int_arg(&in, N_page_size, 0, &a.page_size))
    return NULL;
  if (data(get(&in, N_n_vis), &a.n_vis) || data_attr(out, N_n_vis_out, &a.n_vis_out) || data_attr(out, N_grp_off, &a.grp_off) ||
      data_attr(out, N_grp_src, &a.grp_src) || data_attr(out, N_weight, &a.weight) || data_attr(out, N_status, &a.status) ||
      data(in.v[N_k_src], &a.k_src) || data(in.v[N_v_src], &a.v_src) || data(in.v[N_k_dst], &a.k_dst) ||
      data(in.v[N_v_dst], &a.v_dst) || strides(in.v[N_k_src], 3, s[0]) || strides(in.v[N_v_src], 3, s[1]) ||
      strides(in.v[N_k_dst], 3, s[2]) || strides(in.v[N_v_dst], 3, s[3]))
    return NULL;
  if (memcmp(s[0], s[1], sizeof(s[0])) || memcmp(s[2], s[3], sizeof(s[2]))) {
    PyErr_SetString(PyExc_AssertionError, "K and V have the same strides on either side");
    return NULL;
  }
  a.src_head_stride = s[0][1]; a.src_row_stride = s[0][2];
  a.dst_head_stride = s[2][1]; a.dst_row_stride = s[2][2];
  if (a.page_size > 0) {
    PyObject *ts = in.v[N_src_block_table], *td = in.v[N_dst_block_table];
    int32_t blocks = 0;
    if (!ts || !td) { PyErr_SetString(PyExc_TypeError, "paged caches need src_block_table and dst_block_table"); return NULL; }
    a.src_page_stride = s[0][0]; a.dst_page_stride = s[2][0];
    if (data(ts, &a.src_block_table) || data(td, &a.dst_block_table) || size_of(ts, 1, &a.max_blocks) || size_of(td, 1, &blocks)) return NULL;
    if (blocks != a.max_blocks) { PyErr_SetString(PyExc_AssertionError, "the block tables have the same width"); return NULL; }
  } else {
    a.src_batch_stride = s[0][0]; a.dst_batch_stride = s[2][0];
  }
  if (stream_handle(get(&in, N_stream), &a.stream)) return NULL;
  /* packed caches: sample b's first token; contiguous batch strides become 0 */
  if (get(&in, N_src_seq_start)) { if (data(get(&in, N_src_seq_start), &a.src_seq_start)) return NULL; a.src_batch_stride = 0; }
  if (get(&in, N_dst_seq_start)) { if (data(get(&in, N_dst_seq_start), &a.dst_seq_start)) return NULL; a.dst_batch_stride = 0; }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_kv(plan, &a);
  Py_END_ALLOW_THREADS
  return done(rc, "lightkv_compact_kv");
}

/* ---- serving a compacted cache: these calls take their sizes from the tensors, which are checked here ---- */

typedef struct { int64_t size[4], stride[4]; } View;

/* a tensor on the current device (`device`) of this type and number of dimensions (0: any) -> address, sizes, strides; 16-bit
 * and 32-bit floats when `dtype` is NULL */
static int view(PyObject* t, int id, PyObject* dtype, int dims, long device, void* ptr, View* r) {
  PyObject* v = PyObject_CallMethodNoArgs(t, g_name[N_get_device]);
  if (!v) return -1;
  const long where = PyLong_AsLong(v);
  Py_DECREF(v);
  if (where == -1 && PyErr_Occurred()) return -1;
  if (where != device) {
    PyErr_Format(PyExc_ValueError, "'%U' is not on the current CUDA device", g_name[id]);
    return -1;
  }
  if (dtype) {
    if (!(v = PyObject_GetAttr(t, g_name[N_dtype]))) return -1;
    const int same = v == dtype;
    Py_DECREF(v);
    if (!same) { PyErr_Format(PyExc_TypeError, "'%U' must be of type %S", g_name[id], dtype); return -1; }
  }
  if (dims) {
    if (!(v = PyObject_GetAttr(t, g_name[N_shape]))) return -1;
    int rc = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == dims ? 0 : -1;
    if (rc) PyErr_Format(PyExc_ValueError, "'%U' must have %d dimensions", g_name[id], dims);
    for (int i = 0; i < dims && !rc; ++i) rc = to_i64(PyTuple_GET_ITEM(v, i), &r->size[i]);
    Py_DECREF(v);
    if (rc || strides(t, dims, r->stride)) return -1;
  }
  return data(t, ptr);
}
/* a contiguous array of `n` elements (n < 0: any number) */
static int array(PyObject* t, int id, PyObject* dtype, int64_t n, long device, void* ptr, int64_t* count) {
  View w;
  if (view(t, id, dtype, 1, device, ptr, &w)) return -1;
  if (w.size[0] > 1 && w.stride[0] != 1) { PyErr_Format(PyExc_ValueError, "'%U' must be contiguous", g_name[id]); return -1; }
  if (n >= 0 && w.size[0] != n) { PyErr_Format(PyExc_ValueError, "'%U' must have %lld elements", g_name[id], (long long)n); return -1; }
  if (count) *count = w.size[0];
  return 0;
}
static int same(int id, int64_t got, int64_t want, const char* what) {
  if (got == want) return 0;
  PyErr_Format(PyExc_ValueError, "'%U' has %lld %s, %lld are expected", g_name[id], (long long)got, what, (long long)want);
  return -1;
}
static int to_i32(int id, int64_t v, int32_t* r) {
  if (v < 0 || v > INT32_MAX) { PyErr_Format(PyExc_OverflowError, "a size of '%U' is out of range", g_name[id]); return -1; }
  *r = (int32_t)v;
  return 0;
}
/* rows are contiguous in their last dimension */
static int rows(int id, const View* w, int last) {
  if (w->size[last] <= 1 || w->stride[last] == 1) return 0;
  PyErr_Format(PyExc_ValueError, "'%U' must be contiguous in its last dimension", g_name[id]);
  return -1;
}
static int float_type(PyObject* t, int id, PyObject** dtype, int32_t* r) {
  PyObject* v = PyObject_GetAttr(t, g_name[N_dtype]);
  if (!v) return -1;
  Py_DECREF(v);                                               /* torch keeps its dtypes */
  *r = v == g_bf16 ? LIGHTKV_BF16 : v == g_fp32 ? LIGHTKV_FP32 : -1;
  *dtype = v;
  if (*r < 0) PyErr_Format(PyExc_TypeError, "'%U' must be bfloat16 or float32", g_name[id]);
  return *r < 0 ? -1 : 0;
}
static int current_device(long* r) {
  PyObject* v = PyObject_CallNoArgs(g_device);
  if (!v) return -1;
  *r = PyLong_AsLong(v);
  Py_DECREF(v);
  return *r == -1 && PyErr_Occurred() ? -1 : 0;
}
/* scratch tensor -> its first 256-byte boundary and the bytes behind that */
static int scratch(PyObject* t, long device, void** ptr, size_t* bytes) {
  void* p;
  if (view(t, N_workspace, NULL, 0, device, &p, NULL)) return -1;
  PyObject* v = PyObject_CallMethodNoArgs(t, g_name[N_is_contiguous]);
  if (!v) return -1;
  const int contiguous = PyObject_IsTrue(v);
  Py_DECREF(v);
  if (contiguous < 0) return -1;
  if (!contiguous) { PyErr_SetString(PyExc_ValueError, "'workspace' must be contiguous"); return -1; }
  if (!(v = PyObject_GetAttr(t, g_name[N_nbytes]))) return -1;
  const size_t n = PyLong_AsSize_t(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) return -1;
  const size_t shift = (size_t)(-(uintptr_t)p & 255);
  *ptr = (void*)((uintptr_t)p + shift);
  *bytes = n > shift ? n - shift : 0;
  return 0;
}
/* K and V caches, pages or samples first: the same shape and strides */
static int caches(const Args* in, PyObject* dtype, long device, void* k, void* v, View* c) {
  View w;
  if (view(in->v[N_k_cache], N_k_cache, dtype, 4, device, k, c) || view(in->v[N_v_cache], N_v_cache, dtype, 4, device, v, &w) ||
      rows(N_k_cache, c, 3) || rows(N_v_cache, &w, 3))
    return -1;
  if (memcmp(c, &w, sizeof(w))) { PyErr_SetString(PyExc_ValueError, "'k_cache' and 'v_cache' must have the same shape and strides"); return -1; }
  return 0;
}
/* new K and V rows [n, H_kv, dh]: the same shape and strides */
static int new_rows(const Args* in, PyObject* dtype, long device, void* k, void* v, int64_t heads, int64_t dh, View* c) {
  View w;
  if (view(in->v[N_k_new], N_k_new, dtype, 3, device, k, c) || view(in->v[N_v_new], N_v_new, dtype, 3, device, v, &w) ||
      rows(N_k_new, c, 2) || rows(N_v_new, &w, 2) || same(N_k_new, c->size[1], heads, "heads") || same(N_k_new, c->size[2], dh, "channels"))
    return -1;
  if (c->size[0] != w.size[0] || c->size[1] != w.size[1] || c->size[2] != w.size[2] || c->stride[0] != w.stride[0] || c->stride[1] != w.stride[1]) {
    PyErr_SetString(PyExc_ValueError, "'k_new' and 'v_new' must have the same shape and strides");
    return -1;
  }
  return 0;
}

static const int kDecodePos[] = {N_q, N_k_cache, N_v_cache, N_n_keys, N_out};
static const int kDecodeKw[] = {N_block_table, N_lse, N_k_new, N_v_new, N_workspace, N_scale, N_max_keys, N_status, N_stream};

static PyObject* decode_attention(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  Args in;
  if (parse(&in, "decode_attention", args, nargs, kwnames, kDecodePos, 5, 5, kDecodeKw, sizeof(kDecodeKw) / sizeof(int), N_workspace)) return NULL;
  lightkv_decode_args_t a;
  memset(&a, 0, sizeof(a));
  a.struct_size = sizeof(a);
  View q, c, w;
  PyObject *dtype, *t;
  long dev;
  if (current_device(&dev) || float_type(in.v[N_q], N_q, &dtype, &a.dtype) || view(in.v[N_q], N_q, NULL, 3, dev, &a.q, &q) || rows(N_q, &q, 2) ||
      view(in.v[N_out], N_out, dtype, 3, dev, &a.out, &w) || rows(N_out, &w, 2) || caches(&in, dtype, dev, &a.k_cache, &a.v_cache, &c))
    return NULL;
  for (int i = 0; i < 3; ++i) if (same(N_out, w.size[i], q.size[i], i == 0 ? "requests" : i == 1 ? "heads" : "channels")) return NULL;
  a.q_batch_stride = q.stride[0]; a.q_head_stride = q.stride[1];
  a.out_batch_stride = w.stride[0]; a.out_head_stride = w.stride[1];
  a.page_stride = c.stride[0]; a.head_stride = c.stride[1]; a.row_stride = c.stride[2];
  if (to_i32(N_q, q.size[0], &a.batch) || to_i32(N_q, q.size[1], &a.n_q_heads) || to_i32(N_k_cache, c.size[1], &a.n_kv_heads) ||
      to_i32(N_q, q.size[2], &a.head_dim) || same(N_k_cache, c.size[3], q.size[2], "channels") ||
      array(in.v[N_n_keys], N_n_keys, g_i32, q.size[0], dev, &a.n_keys, NULL) || int_arg(&in, N_max_keys, 0, &a.max_keys))
    return NULL;
  if ((t = get(&in, N_block_table))) {
    if (view(t, N_block_table, g_i32, 2, dev, &a.block_table, &w) || same(N_block_table, w.size[0], q.size[0], "rows") || rows(N_block_table, &w, 1) ||
        to_i32(N_block_table, w.size[0] > 1 ? w.stride[0] : w.size[1], &a.max_blocks) || to_i32(N_k_cache, c.size[0], &a.n_pages) ||
        to_i32(N_k_cache, c.size[2], &a.page_size))
      return NULL;
    if (a.max_blocks != w.size[1]) { PyErr_SetString(PyExc_ValueError, "'block_table' must be contiguous"); return NULL; }
    if (!a.page_size) { PyErr_SetString(PyExc_ValueError, "'k_cache' has pages without rows"); return NULL; }
  } else if (same(N_k_cache, c.size[0], q.size[0], "requests") || to_i32(N_k_cache, c.size[2], &a.max_keys)) {
    return NULL;
  }
  if ((t = get(&in, N_lse))) {
    if (view(t, N_lse, g_fp32, 2, dev, &a.lse, &w) || same(N_lse, w.size[0], q.size[0], "requests") || same(N_lse, w.size[1], q.size[1], "heads")) return NULL;
    a.lse_batch_stride = w.stride[0]; a.lse_head_stride = w.stride[1];
  }
  if (!get(&in, N_k_new) != !get(&in, N_v_new)) { PyErr_SetString(PyExc_ValueError, "'k_new' and 'v_new' come together"); return NULL; }
  if (get(&in, N_k_new)) {
    if (new_rows(&in, dtype, dev, &a.k_new, &a.v_new, c.size[1], c.size[3], &w) || same(N_k_new, w.size[0], q.size[0], "requests")) return NULL;
    a.new_batch_stride = w.stride[0]; a.new_head_stride = w.stride[1];
  }
  if ((t = get(&in, N_scale))) {
    const double scale = PyFloat_AsDouble(t);
    if (scale == -1.0 && PyErr_Occurred()) return NULL;
    a.scale = (float)scale;
  }
  if ((t = get(&in, N_status)) && array(t, N_status, g_i32, 1, dev, &a.status, NULL)) return NULL;
  if (scratch(in.v[N_workspace], dev, &a.workspace, &a.workspace_bytes) || stream_handle(get(&in, N_stream), &a.stream)) return NULL;
  if (!a.batch) Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_decode(&a);
  Py_END_ALLOW_THREADS
  return done(rc, "lightkv_decode_attention");
}

static const int kAppendPos[] = {N_k_new, N_v_new, N_k_cache, N_v_cache, N_slot_map};
static const int kAppendKw[] = {N_status, N_stream};

static PyObject* append_kv(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  Args in;
  if (parse(&in, "append_kv", args, nargs, kwnames, kAppendPos, 5, 5, kAppendKw, sizeof(kAppendKw) / sizeof(int), N_slot_map)) return NULL;
  lightkv_append_args_t a;
  memset(&a, 0, sizeof(a));
  a.struct_size = sizeof(a);
  View c, w;
  PyObject *dtype, *t;
  long dev;
  if (current_device(&dev) || float_type(in.v[N_k_cache], N_k_cache, &dtype, &a.dtype) ||
      caches(&in, dtype, dev, &a.k_cache, &a.v_cache, &c) ||
      new_rows(&in, dtype, dev, &a.k_new, &a.v_new, c.size[1], c.size[3], &w) ||
      array(in.v[N_slot_map], N_slot_map, g_i64, w.size[0], dev, &a.slot_map, NULL) || to_i32(N_k_new, w.size[0], &a.n_tokens) ||
      to_i32(N_k_cache, c.size[0], &a.n_pages) || to_i32(N_k_cache, c.size[1], &a.n_kv_heads) || to_i32(N_k_cache, c.size[2], &a.page_size) ||
      to_i32(N_k_cache, c.size[3], &a.head_dim))
    return NULL;
  a.new_token_stride = w.stride[0]; a.new_head_stride = w.stride[1];
  a.page_stride = c.stride[0]; a.head_stride = c.stride[1]; a.row_stride = c.stride[2];
  if ((t = get(&in, N_status)) && array(t, N_status, g_i32, 1, dev, &a.status, NULL)) return NULL;
  if (stream_handle(get(&in, N_stream), &a.stream)) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_append(&a);
  Py_END_ALLOW_THREADS
  return done(rc, "lightkv_append_kv");
}

static const int kPagesPos[] = {N_seq_len, N_block_table, N_free_pages, N_n_free};
static const int kPagesKw[] = {N_page_size, N_add, N_held, N_seq_len_out, N_n_free_out, N_slot_map, N_slot_start, N_slot_stride, N_workspace,
                               N_status, N_stream};

static PyObject* assign_pages(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  Args in;
  if (parse(&in, "assign_pages", args, nargs, kwnames, kPagesPos, 4, 4, kPagesKw, sizeof(kPagesKw) / sizeof(int), N_workspace)) return NULL;
  if (!get(&in, N_page_size)) { PyErr_SetString(PyExc_TypeError, "assign_pages() missing 1 required keyword-only argument: 'page_size'"); return NULL; }
  lightkv_pages_args_t a;
  memset(&a, 0, sizeof(a));
  a.struct_size = sizeof(a);
  View w;
  PyObject* t;
  long dev;
  int64_t batch, pages, slots = 0;
  if (current_device(&dev) || array(in.v[N_seq_len], N_seq_len, g_i32, -1, dev, &a.seq_len, &batch) ||
      view(in.v[N_block_table], N_block_table, g_i32, 2, dev, &a.block_table, &w) || same(N_block_table, w.size[0], batch, "rows") ||
      rows(N_block_table, &w, 1) || array(in.v[N_free_pages], N_free_pages, g_i32, -1, dev, &a.free_pages, &pages) ||
      array(in.v[N_n_free], N_n_free, g_i32, 1, dev, &a.n_free, NULL) || to_i32(N_seq_len, batch, &a.batch) ||
      to_i32(N_free_pages, pages, &a.n_pages) || to_i32(N_block_table, w.size[1], &a.max_blocks) ||
      int_arg(&in, N_page_size, 0, &a.page_size) || int_arg(&in, N_add, 0, &a.add) || int_arg(&in, N_slot_stride, 0, &a.slot_stride))
    return NULL;
  if (w.size[0] > 1 && w.stride[0] != w.size[1]) { PyErr_SetString(PyExc_ValueError, "'block_table' must be contiguous"); return NULL; }
  if ((t = get(&in, N_held)) && array(t, N_held, g_i32, batch, dev, &a.held, NULL)) return NULL;
  /* lengths are replaced in place unless told otherwise: the ones held, or the ones asked for where none are */
  a.seq_len_out = (int32_t*)(a.held ? a.held : a.seq_len);
  a.n_free_out = (int32_t*)a.n_free;
  if ((t = get(&in, N_seq_len_out)) && array(t, N_seq_len_out, g_i32, batch, dev, &a.seq_len_out, NULL)) return NULL;
  if ((t = get(&in, N_n_free_out)) && array(t, N_n_free_out, g_i32, 1, dev, &a.n_free_out, NULL)) return NULL;
  if ((t = get(&in, N_slot_map)) && (array(t, N_slot_map, g_i64, -1, dev, &a.slot_map, &slots) || to_i32(N_slot_map, slots, &a.n_slots))) return NULL;
  if ((t = get(&in, N_slot_start)) && array(t, N_slot_start, g_i32, batch + 1, dev, &a.slot_start, NULL)) return NULL;
  if ((t = get(&in, N_status)) && array(t, N_status, g_i32, 1, dev, &a.status, NULL)) return NULL;
  if (scratch(in.v[N_workspace], dev, &a.workspace, &a.workspace_bytes) || stream_handle(get(&in, N_stream), &a.stream)) return NULL;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_pages(&a);
  Py_END_ALLOW_THREADS
  return done(rc, "lightkv_assign_pages");
}

/* bind((address of lightkv_compress_layer, of lightkv_compress_layer_builtin_ws, of lightkv_compact_kv, of
 *       lightkv_decode_attention, of lightkv_append_kv, of lightkv_assign_pages),
 *      fail(code, what) -> raises, fork_join(out) -> (event, event), raw_stream(device) -> handle, device() -> index,
 *      (bfloat16, float32, int32, int64)) */
static PyObject* bind(PyObject* self, PyObject* args) {
  unsigned long long l, b, k, d, w, p;
  PyObject *fail, *fj, *rs, *dev, *t[4];
  if (!PyArg_ParseTuple(args, "(KKKKKK)OOOO(OOOO)", &l, &b, &k, &d, &w, &p, &fail, &fj, &rs, &dev, &t[0], &t[1], &t[2], &t[3])) return NULL;
  g_layer = (layer_fn)(uintptr_t)l; g_layer_builtin = (layer_fn)(uintptr_t)b; g_kv = (kv_fn)(uintptr_t)k;
  g_decode = (decode_fn)(uintptr_t)d; g_append = (append_fn)(uintptr_t)w; g_pages = (pages_fn)(uintptr_t)p;
  Py_INCREF(fail); Py_INCREF(fj); Py_INCREF(rs); Py_INCREF(dev);
  Py_XSETREF(g_fail, fail); Py_XSETREF(g_fork_join, fj); Py_XSETREF(g_raw_stream, rs); Py_XSETREF(g_device, dev);
  PyObject** keep[4] = {&g_bf16, &g_fp32, &g_i32, &g_i64};
  for (int i = 0; i < 4; ++i) { Py_INCREF(t[i]); Py_XSETREF(*keep[i], t[i]); }
  Py_RETURN_NONE;
}

static PyMethodDef kMethods[] = {
    {"compress_layer", (PyCFunction)(void (*)(void))compress_layer, METH_FASTCALL | METH_KEYWORDS, NULL},
    {"compress_layer_builtin_ws", (PyCFunction)(void (*)(void))compress_layer_builtin_ws, METH_FASTCALL | METH_KEYWORDS, NULL},
    {"compact_kv", (PyCFunction)(void (*)(void))compact_kv, METH_FASTCALL | METH_KEYWORDS, NULL},
    {"decode_attention", (PyCFunction)(void (*)(void))decode_attention, METH_FASTCALL | METH_KEYWORDS, NULL},
    {"append_kv", (PyCFunction)(void (*)(void))append_kv, METH_FASTCALL | METH_KEYWORDS, NULL},
    {"assign_pages", (PyCFunction)(void (*)(void))assign_pages, METH_FASTCALL | METH_KEYWORDS, NULL},
    {"bind", bind, METH_VARARGS, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", NULL, -1, kMethods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__binding(void) {
#define X(n) if (!(g_name[N_##n] = PyUnicode_InternFromString(#n))) return NULL;
  NAMES(X)
#undef X
  if (!(g_stride = PyUnicode_InternFromString("stride"))) return NULL;
  return PyModule_Create(&kModule);
}
