// Argument marshalling of the serving calls of the Python binding (module _serving): decode_attention, append_kv and assign_pages
// take their sizes from the tensors, which are checked here.  These calls are as short as 1.5 us on the GPU and are made for
// every layer of every token, so the tensors are read through torch's C++ classes: ten methods of Python objects
// took 4 us a call, as much as the rest of it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "lightkv.h"

namespace {

int (*g_decode)(const lightkv_decode_args_t*);
int (*g_append)(const lightkv_append_args_t*);
int (*g_pages)(const lightkv_pages_args_t*);
PyObject* g_load;        // load() loads the library and calls bind()
PyObject* g_fail;        // fail(code, what) raises

struct Error {};         // a Python exception is set

[[noreturn]] void refuse(PyObject* type, const char* format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(type, format, args);
  va_end(args);
  throw Error();
}

// names of all arguments, interned once
#define NAMES(X) \
  X(q) X(k_cache) X(v_cache) X(n_keys) X(out) X(block_table) X(lse) X(k_new) X(v_new) X(workspace) X(scale) X(max_keys) X(status) X(stream) \
  X(slot_map) X(seq_len) X(free_pages) X(n_free) X(page_size) X(add) X(held) X(seq_len_out) X(n_free_out) X(slot_start) X(slot_stride)
enum Name {
#define X(n) N_##n,
  NAMES(X)
#undef X
  N_COUNT
};
const char* const kText[] = {
#define X(n) #n,
    NAMES(X)
#undef X
};
PyObject* g_name[N_COUNT];
PyObject* g_cuda_stream;

// The arguments of a call: `n_positional` names that may be given by position and must be there, further keywords of which the
// first `n_needed` must be there.
struct Args {
  PyObject* v[N_COUNT] = {};
  const char* fn;
  Args(const char* name, PyObject* const* args, Py_ssize_t n, PyObject* kwnames, const Name* names, int n_positional, int n_needed, int n_names)
      : fn(name) {
    if (n > n_positional) refuse(PyExc_TypeError, "%s() takes %d positional arguments but %zd were given", fn, n_positional, n);
    for (Py_ssize_t i = 0; i < n; ++i) v[names[i]] = args[i];
    const Py_ssize_t n_kw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t i = 0; i < n_kw; ++i) {
      PyObject* word = PyTuple_GET_ITEM(kwnames, i);
      int id = -1;
      for (int j = n_names - 1; j >= 0 && id < 0; --j)       // interned names are equal as pointers
        if (word == g_name[names[j]]) id = names[j];
      for (int j = 0; j < n_names && id < 0; ++j)
        if (PyUnicode_Compare(word, g_name[names[j]]) == 0) id = names[j];
      if (id < 0) refuse(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", fn, word);
      if (v[id]) refuse(PyExc_TypeError, "%s() got multiple values for argument '%U'", fn, word);
      v[id] = args[n + i];
    }
    for (int j = 0; j < n_positional + n_needed; ++j)
      if (!v[names[j]]) refuse(PyExc_TypeError, "%s() missing required argument: '%s'", fn, kText[names[j]]);
  }
  PyObject* get(Name id) const { return v[id] == Py_None ? nullptr : v[id]; }

  int32_t integer(Name id, int32_t fallback) const {
    PyObject* o = get(id);
    if (!o) return fallback;
    const long long x = PyLong_AsLongLong(o);                // (also what has __index__)
    if (x == -1 && PyErr_Occurred()) throw Error();
    if (x < INT32_MIN || x > INT32_MAX) refuse(PyExc_OverflowError, "'%s' is out of range", kText[id]);
    return int32_t(x);
  }

  // a tensor on the current device, of `dims` dimensions (0: any) and type `type` (Undefined: any)
  const at::Tensor& tensor(Name id, int dims, at::ScalarType type) const {
    if (!v[id] || !THPVariable_Check(v[id])) refuse(PyExc_TypeError, "'%s' must be a tensor", kText[id]);
    const at::Tensor& t = THPVariable_Unpack(v[id]);
    if (!t.is_cuda() || t.get_device() != c10::cuda::current_device()) refuse(PyExc_ValueError, "'%s' is not on the current CUDA device", kText[id]);
    if (t.layout() != at::kStrided) refuse(PyExc_ValueError, "'%s' must be strided", kText[id]);
    if (type != at::ScalarType::Undefined && t.scalar_type() != type) refuse(PyExc_TypeError, "'%s' must be of type %s", kText[id], c10::toString(type));
    if (dims && t.dim() != dims) refuse(PyExc_ValueError, "'%s' must have %d dimensions", kText[id], dims);
    return t;
  }
  // ... whose last dimension is contiguous
  const at::Tensor& rows(Name id, int dims, at::ScalarType type) const {
    const at::Tensor& t = tensor(id, dims, type);
    if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) refuse(PyExc_ValueError, "'%s' must be contiguous in its last dimension", kText[id]);
    return t;
  }
  // a contiguous array of n elements (n < 0: any number)
  template <typename T>
  T* array(Name id, at::ScalarType type, int64_t n, int64_t* count = nullptr) const {
    const at::Tensor& t = rows(id, 1, type);
    if (n >= 0) same(id, t.size(0), n, "elements");
    if (count) *count = t.size(0);
    return static_cast<T*>(t.data_ptr());
  }
  static void same(Name id, int64_t got, int64_t want, const char* what) {
    if (got != want) refuse(PyExc_ValueError, "'%s' has %lld %s, %lld are expected", kText[id], (long long)got, what, (long long)want);
  }
  static int32_t size(Name id, int64_t n) {
    if (n < 0 || n > INT32_MAX) refuse(PyExc_OverflowError, "a size of '%s' is out of range", kText[id]);
    return int32_t(n);
  }
  // a block table [batch, blocks]: its row stride, which is its width
  int32_t table(int64_t batch, int32_t** data) const {
    const at::Tensor& t = rows(N_block_table, 2, at::kInt);
    same(N_block_table, t.size(0), batch, "rows");
    if (t.size(0) > 1 && t.stride(0) != t.size(1)) refuse(PyExc_ValueError, "'block_table' must be contiguous");
    *data = static_cast<int32_t*>(t.data_ptr());
    return size(N_block_table, t.size(1));
  }
  // K and V: the same shape and strides
  const at::Tensor& pair(Name k, Name v_id, int dims, at::ScalarType type, void** k_data, void** v_data) const {
    const at::Tensor &a = rows(k, dims, type), &b = rows(v_id, dims, type);
    if (a.sizes() != b.sizes()) refuse(PyExc_ValueError, "'%s' and '%s' must have the same shape", kText[k], kText[v_id]);
    for (int i = 0; i < dims; ++i)
      if (a.size(i) > 1 && a.stride(i) != b.stride(i)) refuse(PyExc_ValueError, "'%s' and '%s' must have the same strides", kText[k], kText[v_id]);
    *k_data = a.data_ptr();
    *v_data = b.data_ptr();
    return a;
  }
  // the first 256-byte boundary of the workspace, and the bytes behind it
  void scratch(void** data, size_t* bytes) const {
    const at::Tensor& t = tensor(N_workspace, 0, at::ScalarType::Undefined);
    if (!t.is_contiguous()) refuse(PyExc_ValueError, "'workspace' must be contiguous");
    const uintptr_t p = reinterpret_cast<uintptr_t>(t.data_ptr()), up = (p + 255) / 256 * 256;
    *data = reinterpret_cast<void*>(up);
    *bytes = t.nbytes() > up - p ? t.nbytes() - (up - p) : 0;
  }
  uint32_t* status() const { return get(N_status) ? array<uint32_t>(N_status, at::kInt, 1) : nullptr; }
  void* stream() const {
    PyObject* s = get(N_stream);
    if (!s) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* handle = PyObject_GetAttr(s, g_cuda_stream);
    if (!handle) throw Error();
    void* p = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!p && PyErr_Occurred()) throw Error();
    return p;
  }
};

// The stride of dimension i; one that holds a single element is never stepped over, whatever stride it has: `alone` then.
int64_t step(const at::Tensor& t, int i, int64_t alone = 0) { return t.size(i) > 1 ? t.stride(i) : alone; }

int32_t float_type(const at::Tensor& t, Name id) {
  if (t.scalar_type() == at::kBFloat16) return LIGHTKV_BF16;
  if (t.scalar_type() == at::kFloat) return LIGHTKV_FP32;
  refuse(PyExc_TypeError, "'%s' must be bfloat16 or float32", kText[id]);
}

void loaded() {
  if (g_pages) return;
  if (!g_load) refuse(PyExc_RuntimeError, "_serving has not been set up");
  PyObject* r = PyObject_CallNoArgs(g_load);
  if (!r) throw Error();
  Py_DECREF(r);
}

template <typename A>
PyObject* call(int (*entry)(const A*), const A& a, const char* what) {
  int code;
  Py_BEGIN_ALLOW_THREADS
  code = entry(&a);
  Py_END_ALLOW_THREADS
  if (code == LIGHTKV_OK) Py_RETURN_NONE;
  return PyObject_CallFunction(g_fail, "is", code, what);    // raises LightKVError
}

// no C++ exception leaves a function that Python calls
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Error&) {
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* decode_attention(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kwnames) {
  return guarded([&]() -> PyObject* {
    static const Name names[] = {N_q, N_k_cache, N_v_cache, N_n_keys, N_out, N_workspace, N_block_table, N_lse, N_k_new, N_v_new, N_slot_map, N_scale,
                                 N_max_keys, N_status, N_stream};
    const Args in("decode_attention", args, n, kwnames, names, 5, 1, 15);
    lightkv_decode_args_t a = {};
    a.struct_size = sizeof(a);
    const at::Tensor& q = in.rows(N_q, 3, at::ScalarType::Undefined);
    a.dtype = float_type(q, N_q);
    const at::ScalarType type = q.scalar_type();
    const at::Tensor& out = in.rows(N_out, 3, type);
    static const char* const what[] = {"requests", "heads", "channels"};
    for (int i = 0; i < 3; ++i) Args::same(N_out, out.size(i), q.size(i), what[i]);
    const at::Tensor& c = in.pair(N_k_cache, N_v_cache, 4, type, &a.k_cache, &a.v_cache);
    Args::same(N_k_cache, c.size(3), q.size(2), what[2]);
    a.batch = Args::size(N_q, q.size(0)); a.n_q_heads = Args::size(N_q, q.size(1)); a.head_dim = Args::size(N_q, q.size(2));
    a.n_kv_heads = Args::size(N_k_cache, c.size(1));
    a.q = q.data_ptr(); a.q_batch_stride = step(q, 0); a.q_head_stride = step(q, 1);
    a.out = out.data_ptr(); a.out_batch_stride = step(out, 0); a.out_head_stride = step(out, 1);
    a.page_stride = step(c, 0); a.head_stride = step(c, 1); a.row_stride = step(c, 2, c.size(3));
    a.n_keys = in.array<int32_t>(N_n_keys, at::kInt, q.size(0));
    a.max_keys = in.integer(N_max_keys, 0);
    if (in.get(N_block_table)) {
      int32_t* table;
      a.max_blocks = in.table(q.size(0), &table);
      a.block_table = table;
      a.n_pages = Args::size(N_k_cache, c.size(0));
      a.page_size = Args::size(N_k_cache, c.size(2));
      if (!a.page_size) refuse(PyExc_ValueError, "'k_cache' has pages without rows");
    } else {
      Args::same(N_k_cache, c.size(0), q.size(0), what[0]);
      a.key_bound = a.max_keys;
      a.max_keys = Args::size(N_k_cache, c.size(2));
    }
    if (in.get(N_lse)) {
      const at::Tensor& t = in.tensor(N_lse, 2, at::kFloat);
      for (int i = 0; i < 2; ++i) Args::same(N_lse, t.size(i), q.size(i), what[i]);
      a.lse = static_cast<float*>(t.data_ptr()); a.lse_batch_stride = t.stride(0); a.lse_head_stride = t.stride(1);
    }
    if (!in.get(N_k_new) != !in.get(N_v_new)) refuse(PyExc_ValueError, "'k_new' and 'v_new' come together");
    if (in.get(N_k_new)) {
      void *k, *v;
      const at::Tensor& t = in.pair(N_k_new, N_v_new, 3, type, &k, &v);
      Args::same(N_k_new, t.size(0), q.size(0), what[0]);
      Args::same(N_k_new, t.size(1), c.size(1), what[1]);
      Args::same(N_k_new, t.size(2), c.size(3), what[2]);
      a.k_new = k; a.v_new = v; a.new_batch_stride = step(t, 0); a.new_head_stride = step(t, 1);
    }
    if (in.get(N_slot_map)) {
      if (!a.k_new) refuse(PyExc_ValueError, "'slot_map' comes with 'k_new' and 'v_new'");
      a.slot_map = in.array<int64_t>(N_slot_map, at::kLong, q.size(0));
    }
    if (PyObject* s = in.get(N_scale)) {
      const double scale = PyFloat_AsDouble(s);
      if (scale == -1.0 && PyErr_Occurred()) throw Error();
      a.scale = float(scale);
    }
    a.status = in.status();
    in.scratch(&a.workspace, &a.workspace_bytes);
    a.stream = in.stream();
    if (!a.batch) Py_RETURN_NONE;
    loaded();
    return call(g_decode, a, "lightkv_decode_attention");
  });
}

PyObject* append_kv(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kwnames) {
  return guarded([&]() -> PyObject* {
    static const Name names[] = {N_k_new, N_v_new, N_k_cache, N_v_cache, N_slot_map, N_status, N_stream};
    const Args in("append_kv", args, n, kwnames, names, 5, 0, 7);
    lightkv_append_args_t a = {};
    a.struct_size = sizeof(a);
    const at::Tensor& first = in.rows(N_k_cache, 4, at::ScalarType::Undefined);
    a.dtype = float_type(first, N_k_cache);
    const at::Tensor& c = in.pair(N_k_cache, N_v_cache, 4, first.scalar_type(), &a.k_cache, &a.v_cache);
    void *k, *v;
    const at::Tensor& t = in.pair(N_k_new, N_v_new, 3, first.scalar_type(), &k, &v);
    Args::same(N_k_new, t.size(1), c.size(1), "heads");
    Args::same(N_k_new, t.size(2), c.size(3), "channels");
    a.k_new = k; a.v_new = v; a.new_token_stride = step(t, 0); a.new_head_stride = step(t, 1);
    a.slot_map = in.array<int64_t>(N_slot_map, at::kLong, t.size(0));
    a.n_tokens = Args::size(N_k_new, t.size(0)); a.n_pages = Args::size(N_k_cache, c.size(0)); a.n_kv_heads = Args::size(N_k_cache, c.size(1));
    a.page_size = Args::size(N_k_cache, c.size(2)); a.head_dim = Args::size(N_k_cache, c.size(3));
    a.page_stride = step(c, 0); a.head_stride = step(c, 1); a.row_stride = step(c, 2, c.size(3));
    a.status = in.status();
    a.stream = in.stream();
    loaded();
    return call(g_append, a, "lightkv_append_kv");
  });
}

PyObject* assign_pages(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kwnames) {
  return guarded([&]() -> PyObject* {
    static const Name names[] = {N_seq_len, N_block_table, N_free_pages, N_n_free, N_page_size, N_workspace, N_add, N_held, N_seq_len_out, N_n_free_out,
                                 N_slot_map, N_slot_start, N_slot_stride, N_status, N_stream};
    const Args in("assign_pages", args, n, kwnames, names, 4, 2, 15);
    lightkv_pages_args_t a = {};
    a.struct_size = sizeof(a);
    int64_t batch, pages, slots = 0;
    int32_t* seq_len = in.array<int32_t>(N_seq_len, at::kInt, -1, &batch);
    int32_t* n_free = in.array<int32_t>(N_n_free, at::kInt, 1);
    int32_t* held = in.get(N_held) ? in.array<int32_t>(N_held, at::kInt, batch) : nullptr;
    a.seq_len = seq_len; a.n_free = n_free; a.held = held;
    a.batch = Args::size(N_seq_len, batch);
    a.max_blocks = in.table(batch, &a.block_table);
    a.free_pages = in.array<int32_t>(N_free_pages, at::kInt, -1, &pages);
    a.n_pages = Args::size(N_free_pages, pages);
    if (!in.get(N_page_size)) refuse(PyExc_TypeError, "assign_pages() missing required argument: 'page_size'");
    a.page_size = in.integer(N_page_size, 0); a.add = in.integer(N_add, 0); a.slot_stride = in.integer(N_slot_stride, 0);
    // lengths are replaced in place unless told otherwise: the ones held, or the ones asked for where none are
    a.seq_len_out = in.get(N_seq_len_out) ? in.array<int32_t>(N_seq_len_out, at::kInt, batch) : held ? held : seq_len;
    a.n_free_out = in.get(N_n_free_out) ? in.array<int32_t>(N_n_free_out, at::kInt, 1) : n_free;
    if (in.get(N_slot_map)) {
      a.slot_map = in.array<int64_t>(N_slot_map, at::kLong, -1, &slots);
      a.n_slots = Args::size(N_slot_map, slots);
    }
    if (in.get(N_slot_start)) a.slot_start = in.array<int32_t>(N_slot_start, at::kInt, batch + 1);
    a.status = in.status();
    in.scratch(&a.workspace, &a.workspace_bytes);
    a.stream = in.stream();
    loaded();
    return call(g_pages, a, "lightkv_assign_pages");
  });
}

// setup(load, fail): load() loads the library and calls bind(); fail(code, what) raises
PyObject* setup(PyObject*, PyObject* args) {
  PyObject *load, *fail;
  if (!PyArg_ParseTuple(args, "OO", &load, &fail)) return nullptr;
  Py_INCREF(load); Py_INCREF(fail);
  Py_XSETREF(g_load, load); Py_XSETREF(g_fail, fail);
  Py_RETURN_NONE;
}

// bind(addresses of lightkv_decode_attention, lightkv_append_kv, lightkv_assign_pages)
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long d, w, p;
  if (!PyArg_ParseTuple(args, "KKK", &d, &w, &p)) return nullptr;
  g_decode = reinterpret_cast<decltype(g_decode)>(uintptr_t(d));
  g_append = reinterpret_cast<decltype(g_append)>(uintptr_t(w));
  g_pages = reinterpret_cast<decltype(g_pages)>(uintptr_t(p));
  Py_RETURN_NONE;
}

#define METHOD(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f))
PyMethodDef kMethods[] = {
    {"decode_attention", METHOD(decode_attention), METH_FASTCALL | METH_KEYWORDS,
     "decode_attention(q, k_cache, v_cache, n_keys, out, *, workspace, block_table=None, lse=None, k_new=None, v_new=None,\n"
     "                 slot_map=None, scale=None, max_keys=0, status=None, stream=None)\n\n"
     "lightkv_decode_attention.  q, out [B,H,dh]; n_keys [B] int32.  With block_table [B,max_blocks] int32 the caches are page pools\n"
     "[n_pages,H_kv,page_size,dh], else [B,H_kv,N,dh] (any strides with a contiguous last dimension, the same for K and V).\n"
     "workspace: a tensor of decode_workspace_bytes bytes; lse [B,H] fp32; k_new / v_new [B,H_kv,dh]: rows that stand for key\n"
     "n_keys - 1 and are written to the cache; slot_map [B] int64 (as assign_pages writes it with slot_stride=1): a request whose\n"
     "entry is negative has no new row, and its n_keys rows are read as they stand; scale: None or 0 for 1 / sqrt(dh); max_keys: an\n"
     "upper bound of n_keys, by which the split of the work is chosen (0: all rows that the table or the cache has room for);\n"
     "status [1] int32.  All tensors are on the current device.  No requests: nothing happens."},
    {"append_kv", METHOD(append_kv), METH_FASTCALL | METH_KEYWORDS,
     "append_kv(k_new, v_new, k_cache, v_cache, slot_map, *, status=None, stream=None)\n\n"
     "lightkv_append_kv.  k_new, v_new [T,H_kv,dh]; caches [n_pages,H_kv,page_size,dh]; slot_map [T] int64, negative: skipped;\n"
     "status [1] int32."},
    {"assign_pages", METHOD(assign_pages), METH_FASTCALL | METH_KEYWORDS,
     "assign_pages(seq_len, block_table, free_pages, n_free, *, page_size, workspace, add=0, held=None, seq_len_out=None,\n"
     "             n_free_out=None, slot_map=None, slot_start=None, slot_stride=0, status=None, stream=None)\n\n"
     "lightkv_assign_pages.  seq_len [B], block_table [B,max_blocks], free_pages [n_pages], n_free [1]: int32.  workspace: a tensor of\n"
     "pages_workspace_bytes bytes; held [B] int32; seq_len_out [B] (default: in place of held, or of seq_len where none is given);\n"
     "n_free_out [1] (default: in place of n_free); slot_map [n_slots] int64; slot_start [B+1] int32; status [1] int32.  A batch of\n"
     "no requests is refused."},
    {"setup", METHOD(setup), METH_VARARGS, nullptr},
    {"bind", METHOD(bind), METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving() {
  for (int i = 0; i < N_COUNT; ++i)
    if (!(g_name[i] = PyUnicode_InternFromString(kText[i]))) return nullptr;
  if (!(g_cuda_stream = PyUnicode_InternFromString("cuda_stream"))) return nullptr;
  return PyModule_Create(&kModule);
}
