// Argument marshalling of the hot calls of the Python binding (module _ptdcall).
//
// A call through ctypes cost 7-10 us of host time beside the launch itself (Python-level checks
// of every tensor, torch.cuda.current_stream(), the conversion of a dozen arguments), more
// than many of the kernels take.  Each function here takes the same arguments as its
// counterpart in ptd.py, makes the same checks (a CUDA tensor, contiguous, of the right dtype) and
// calls the C ABI function.  It returns the number of kernels launched, or minus the status
// when the library refuses the call, or None when an argument is not of the plain form
// expected here: nothing has been enqueued then, and ptd.py's own path handles the call or
// raises its error.  Nothing is kept between calls.
//
// A torch.Tensor is looked at through torch's own C++ class (an attribute read by name costs 0.07 - 0.16 us, and a call has up
// to a dozen tensors with five or six each: prompt_norm_rope_append 3.0 us without the launch); an object of another type that load() was
// given by its Python attributes.  That class is the one of the torch compiled against: load() refuses another version.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "../../include/ptd.h"

namespace {

PyObject *g_tensor, *g_i32, *g_f32, *g_bf16, *g_raw_stream, *g_get_device;
PyObject *s_is_cuda, *s_is_contiguous, *s_dtype, *s_data_ptr, *s_nbytes, *s_shape, *s_stride, *s_c, *s_get_device, *s_k,
    *s_block_table, *s_sizes, *s_ctx_lens;

#define PTD_FUNCTIONS(X)                                                                                            \
  X(ptd_tree_attention) X(ptd_topk_draft) X(ptd_verify_greedy) X(ptd_kv_compact) X(ptd_verify_sampling)             \
  X(ptd_verify_and_compact) X(ptd_draft_tree_update) X(ptd_pool_merge) X(ptd_pool_retrieve) X(ptd_tree_rope_append) \
  X(ptd_lm_head_topk) X(ptd_tree_verify_step) X(ptd_prompt_slots) X(ptd_prompt_rope_append) X(ptd_prompt_attention)   \
  X(ptd_prompt_norm_rope_append) X(ptd_tree_norm_rope_append) X(ptd_token_logprobs) X(ptd_lm_head_logprobs)          \
  X(ptd_page_fork) X(ptd_last_launch_count)
#define PTD_DECLARE(f) decltype(&f) p_##f;
PTD_FUNCTIONS(PTD_DECLARE)
#undef PTD_DECLARE

bool g_direct = false;   // g_tensor is torch.Tensor

// What the calls ask of an object of type g_tensor.  Whatever fails, on the Python side or as a C++ exception, is
// an answer that no call takes (nullptr, -1 or false), with no Python error left.
namespace look {

const at::Tensor& direct(PyObject* o) { return THPVariable_Unpack(o); }

bool truth(PyObject* r) {   // (True outlives the reference dropped here)
  Py_XDECREF(r);
  if (r == nullptr) PyErr_Clear();
  return r == Py_True;
}
int64_t number(PyObject* r) {
  const int64_t v = r != nullptr && PyLong_CheckExact(r) ? PyLong_AsLongLong(r) : -1;
  Py_XDECREF(r);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return -1;
  }
  return v;
}
// the numbers of a tuple of at most four, how many there are
int numbers(PyObject* r, int64_t (&v)[4]) {
  int n = -1;
  if (r != nullptr && PyTuple_Check(r) && PyTuple_GET_SIZE(r) <= 4) {
    n = (int)PyTuple_GET_SIZE(r);
    for (int i = 0; i < n; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(r, i));
  }
  Py_XDECREF(r);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return -1;
  }
  return n;
}
int numbers(at::IntArrayRef a, int64_t (&v)[4]) {
  if (a.size() > 4) return -1;
  for (size_t i = 0; i < a.size(); ++i) v[i] = a[i];
  return (int)a.size();
}

bool is_cuda(PyObject* o) {
  try {
    return g_direct ? direct(o).is_cuda() : truth(PyObject_GetAttr(o, s_is_cuda));
  } catch (...) {
    return false;
  }
}
int64_t device(PyObject* o) {   // -1: not on one
  try {
    return g_direct ? (direct(o).is_cuda() ? direct(o).get_device() : -1) : number(PyObject_CallMethodNoArgs(o, s_get_device));
  } catch (...) {
    return -1;
  }
}
bool is_contiguous(PyObject* o) {
  try {
    return g_direct ? direct(o).is_contiguous() : truth(PyObject_CallMethodNoArgs(o, s_is_contiguous));
  } catch (...) {
    return false;
  }
}
// whether the dtype is this one of int32, float32 and bfloat16
bool has_dtype(PyObject* o, PyObject* dtype) {
  if (g_direct) {
    const auto want = dtype == g_i32 ? at::kInt : (dtype == g_f32 ? at::kFloat : at::kBFloat16);
    return direct(o).scalar_type() == want;
  }
  PyObject* d = PyObject_GetAttr(o, s_dtype);   // (the dtypes outlive the reference dropped here)
  Py_XDECREF(d);
  if (d == nullptr) PyErr_Clear();
  return d == dtype;
}
// false: the tensor has no address
bool address(PyObject* o, void** p) {
  *p = nullptr;
  try {
    if (g_direct) {
      *p = direct(o).data_ptr();
      return true;
    }
  } catch (...) {
    return false;
  }
  PyObject* r = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (r != nullptr) *p = PyLong_AsVoidPtr(r);
  Py_XDECREF(r);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return r != nullptr;
}
int64_t nbytes(PyObject* o) {
  try {
    return g_direct ? direct(o).numel() * (int64_t)direct(o).element_size() : number(PyObject_GetAttr(o, s_nbytes));
  } catch (...) {
    return -1;
  }
}
int shape(PyObject* o, int64_t (&d)[4]) {
  try {
    return g_direct ? numbers(direct(o).sizes(), d) : numbers(PyObject_GetAttr(o, s_shape), d);
  } catch (...) {
    return -1;
  }
}
// the size of dimension i of one with two or more
int64_t named_size(PyObject* o, int i) {
  PyObject* d = PyObject_GetAttr(o, s_shape);
  int64_t n = -1;
  if (d != nullptr && PyTuple_Check(d) && PyTuple_GET_SIZE(d) >= 2) n = PyLong_AsLongLong(PyTuple_GET_ITEM(d, i));
  Py_XDECREF(d);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return -1;
  }
  return n;
}
int64_t size(PyObject* o, int i) {
  try {
    return g_direct ? (direct(o).dim() >= 2 ? direct(o).size(i) : -1) : named_size(o, i);
  } catch (...) {
    return -1;
  }
}
int strides(PyObject* o, int64_t (&d)[4]) {
  try {
    return g_direct ? numbers(direct(o).strides(), d) : numbers(PyObject_CallMethodNoArgs(o, s_stride), d);
  } catch (...) {
    return -1;
  }
}

}  // namespace look

// Reads one call's arguments; the first that is not of the expected form clears `ok`.
struct Args {
  PyObject* const* a;
  Py_ssize_t n, i = 0;
  bool ok = true;
  PyObject* kept[3] = {};   // the structures read, held until the call has returned
  int n_kept = 0;
  Args(PyObject* const* args, Py_ssize_t count, Py_ssize_t want) : a(args), n(count) {
    ok = count == want && g_tensor != nullptr;
  }
  ~Args() {
    while (n_kept > 0) Py_DECREF(kept[--n_kept]);
  }
  Args(const Args&) = delete;
  Args& operator=(const Args&) = delete;
  void fail() {
    ok = false;
    PyErr_Clear();
  }
  PyObject* next() { return a[i++]; }
  bool is_tensor(PyObject* o) { return (PyObject*)Py_TYPE(o) == g_tensor; }
  void* pointer(PyObject* o) {
    void* p;
    if (!look::address(o, &p)) fail();
    return p;
  }
  // a contiguous CUDA tensor of `dtype` (NULL: any)
  void* tensor_of(PyObject* o, PyObject* dtype) {
    if (!ok) return nullptr;
    if (!is_tensor(o) || !look::is_cuda(o) || !look::is_contiguous(o) || (dtype != nullptr && !look::has_dtype(o, dtype))) {
      fail();
      return nullptr;
    }
    return pointer(o);
  }
  // as tensor_of, on the device of the tensors seen by on() (which tells a host tensor too)
  void* tensor_on(PyObject* o, PyObject* dtype) {
    on(o);
    if (!ok) return nullptr;
    if (!look::is_contiguous(o) || (dtype != nullptr && !look::has_dtype(o, dtype))) {
      fail();
      return nullptr;
    }
    return pointer(o);
  }
  void* tensor(PyObject* dtype = nullptr) {
    PyObject* o = next();
    return tensor_of(o, dtype);
  }
  int32_t* i32() { return static_cast<int32_t*>(tensor(g_i32)); }
  float* f32() { return static_cast<float*>(tensor(g_f32)); }
  // None, or a tensor and its size in bytes
  void* optional(size_t* bytes) {
    *bytes = 0;
    PyObject* o = next();
    if (o == Py_None) return nullptr;
    void* p = tensor_of(o, nullptr);
    if (!ok) return nullptr;
    const int64_t n = look::nbytes(o);
    if (n < 0) fail(); else *bytes = (size_t)n;
    return p;
  }
  // the dtype of a bf16 or fp32 tensor
  ptd_dtype kind(PyObject* o) {
    if (!ok) return PTD_F32;
    const bool bf16 = is_tensor(o) && look::has_dtype(o, g_bf16);
    if (!bf16 && !(is_tensor(o) && look::has_dtype(o, g_f32))) fail();
    return bf16 ? PTD_BF16 : PTD_F32;
  }
  // the sizes of a 2-D tensor
  void dims2(PyObject* o, int64_t* d0, int64_t* d1) {
    *d0 = *d1 = 0;
    int64_t d[4];
    if (!ok || !is_tensor(o) || look::shape(o, d) != 2) {
      fail();
      return;
    }
    *d0 = d[0], *d1 = d[1];
  }
  // a 2-D tensor's rows: CUDA, unit column stride, rows at least a row apart
  void* rows2(PyObject* o, PyObject* dtype, int64_t* rows, int64_t* cols, int64_t* stride) {
    *stride = 0;
    dims2(o, rows, cols);
    int64_t st[4];
    if (!ok || !look::is_cuda(o) || !look::has_dtype(o, dtype) || look::strides(o, st) != 2 || st[1] != 1 || st[0] < *cols) {
      fail();
      return nullptr;
    }
    *stride = st[0];
    return pointer(o);
  }
  // The device of the tensors seen by on(): the prompt calls run on it only where it is the current one.
  int64_t device = -1;
  void on(PyObject* o) {
    if (!ok) return;
    const int64_t d = is_tensor(o) ? look::device(o) : -1;
    if (d < 0 || (device >= 0 && d != device)) fail();
    device = d;
  }
  void on_attr(PyObject* o, PyObject* name) {
    if (!ok) return;
    PyObject* t = PyObject_GetAttr(o, name);
    if (t == nullptr) fail(); else on(t);
    Py_XDECREF(t);
  }
  void on_current() {
    if (!ok) return;
    PyObject* d = PyObject_CallNoArgs(g_get_device);
    if (d == nullptr || !PyLong_CheckExact(d) || PyLong_AsLongLong(d) != device) fail();
    Py_XDECREF(d);
  }
  // The batch is the contiguous cache's, or has a row each in its block table (a batch below 1 is the library's to refuse).
  void batch_of(PyObject* o, const ptd_prompt* prompt, const ptd_kv_cache* cache) {
    if (!ok || prompt->batch < 1) return;
    const bool paged = cache->page_size > 0;
    PyObject* t = PyObject_GetAttr(o, paged ? s_block_table : s_k);
    const int64_t rows = t == nullptr ? -1 : (is_tensor(t) ? look::size(t, paged ? 0 : 1) : look::named_size(t, paged ? 0 : 1));
    Py_XDECREF(t);
    if (PyErr_Occurred() || (paged ? rows < prompt->batch : rows != prompt->batch)) fail();
  }
  // a tensor of `count` elements of 32 bits, an int32 one
  void* word_of(PyObject* dtype, int64_t count) {
    PyObject* o = next();
    if (!ok) return nullptr;
    void* p = tensor_on(o, dtype);
    if (!ok || look::nbytes(o) != 4 * count) fail();
    return p;
  }
  int32_t* i32_of(int64_t count) { return static_cast<int32_t*>(word_of(g_i32, count)); }
  // the sizes of a tensor of 2 to 4 dimensions; how many there are
  int dims(PyObject* o, int64_t (&d)[4]) {
    d[0] = d[1] = d[2] = d[3] = 0;
    const int n = ok && is_tensor(o) ? look::shape(o, d) : -1;
    if (n < 1) fail();
    return n;
  }
  // a contiguous tensor of `dtype`, of this shape
  void* shaped(PyObject* dtype, int n, const int64_t* want) {
    PyObject* o = next();
    if (!ok) return nullptr;
    void* p = tensor_on(o, dtype);
    int64_t d[4];
    if (dims(o, d) != n) ok = false;
    for (int i = 0; i < n; ++i) ok = ok && d[i] == want[i];
    return p;
  }
  // log probabilities: tokens, out_logprob, out_entropy (or None), out_idx and out_val (or None) of `rows` rows
  struct Logprobs {
    const int32_t* tokens;
    float *logprob, *entropy, *val;
    int32_t* idx;
    int32_t k;
  };
  Logprobs logprobs(int64_t rows) {
    Logprobs x = {};
    x.tokens = i32_of(rows);
    x.logprob = static_cast<float*>(word_of(g_f32, rows));
    x.entropy = a[i] == Py_None ? (next(), nullptr) : static_cast<float*>(word_of(g_f32, rows));
    if (ok && a[i] == Py_None && a[i + 1] == Py_None) {
      i += 2;
      return x;
    }
    int64_t want[4] = {rows, 0, 0, 0}, k = 0;
    dims2(a[i], &want[0], &k);
    if (want[0] != rows || k < 1 || k > PTD_MAX_TOPK) ok = false;
    want[1] = k;
    x.k = (int32_t)k;
    x.idx = static_cast<int32_t*>(shaped(g_i32, 2, want));
    x.val = static_cast<float*>(shaped(g_f32, 2, want));
    return x;
  }
  // a [rows, heads, dim] tensor whose tokens may be apart, a token's heads back to back (*heads 0: any)
  void* rows3(PyObject* dtype, int64_t rows, int64_t dim, int64_t* heads, int64_t* stride) {
    PyObject* o = next();
    on(o);   // (a host tensor has no device)
    int64_t n[4], st[4];
    if (!ok || !look::has_dtype(o, dtype) || look::shape(o, n) != 3 || look::strides(o, st) != 3 || n[0] != rows || n[2] != dim ||
        n[1] < 1 || (*heads != 0 && n[1] != *heads) || (dim != 1 && st[2] != 1) || (n[1] != 1 && st[1] != dim) || st[0] < n[1] * dim) {
      fail();
      return nullptr;
    }
    *heads = n[1];
    *stride = st[0];
    return pointer(o);
  }
  int64_t i64() {
    PyObject* o = next();
    if (!ok) return 0;
    if (!PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    const int64_t v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) fail();
    return v;
  }
  int32_t num() {
    const int64_t v = i64();
    if (v != (int32_t)v) ok = false;
    return (int32_t)v;
  }
  float real() {
    PyObject* o = next();
    if (!ok) return 0.f;
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) {
      ok = false;
      return 0.f;
    }
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) fail();
    return (float)v;
  }
  // the ctypes structure in the attribute `c` of a Tree, KVCache or StepBuffers (the attribute may be
  // a new object at each read, or be replaced by another thread while the call runs without the lock)
  template <typename S>
  S* structure() {
    PyObject* o = next();
    if (!ok) return nullptr;
    PyObject* c = PyObject_GetAttr(o, s_c);
    Py_buffer v;
    S* p = nullptr;
    if (c != nullptr && PyObject_GetBuffer(c, &v, PyBUF_SIMPLE) == 0) {
      if ((size_t)v.len == sizeof(S) && n_kept < 3) p = static_cast<S*>(v.buf);
      PyBuffer_Release(&v);
    }
    if (p == nullptr) {
      Py_XDECREF(c);
      fail();
      return nullptr;
    }
    kept[n_kept++] = c;
    return p;
  }
  // None (the current stream of the current device) or the stream's address
  void* stream() {
    PyObject* o = next();
    if (!ok) return nullptr;
    if (PyLong_CheckExact(o)) return PyLong_AsVoidPtr(o);
    if (o != Py_None) {
      ok = false;
      return nullptr;
    }
    PyObject* d = PyObject_CallNoArgs(g_get_device);
    PyObject* r = d != nullptr ? PyObject_CallOneArg(g_raw_stream, d) : nullptr;
    void* p = r != nullptr ? PyLong_AsVoidPtr(r) : nullptr;
    Py_XDECREF(d);
    Py_XDECREF(r);
    if (PyErr_Occurred()) fail();
    return p;
  }
};

// The call itself runs without the interpreter lock (a launch can wait for room in the stream).
#define PTD_CALL(expr)          \
  do {                          \
    ptd_status st_;             \
    Py_BEGIN_ALLOW_THREADS      \
    st_ = expr;                 \
    Py_END_ALLOW_THREADS        \
    return done(st_);           \
  } while (0)

PyObject* done(ptd_status st) { return PyLong_FromLong(st == PTD_OK ? (long)p_ptd_last_launch_count() : -(long)st); }

// (tree, cache, layer_begin, num_layers, q, num_q_heads, scale, out, workspace, dev_status, stream)
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 11);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (!g.ok) Py_RETURN_NONE;
  PyObject* dt = cache->dtype == PTD_BF16 ? g_bf16 : g_f32;
  const int32_t l0 = g.num(), nl = g.num();
  const void* q = g.tensor(dt);
  const int32_t hq = g.num();
  const float scale = g.real();
  void* out = g.tensor(dt);
  size_t wsb;
  void* ws = g.optional(&wsb);
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_tree_attention(tree, cache, l0, nl, q, hq, scale, out, ws, wsb, status, s));
}

// (logits, k, out_idx, out_val, vocab, stream)
PyObject* topk_draft(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 6);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_dtype dt = g.kind(a[0]);
  int64_t rows, stride;
  g.dims2(a[0], &rows, &stride);
  const void* logits = g.tensor();
  const int32_t k = g.num();
  int32_t* idx = g.i32();
  float* val = g.f32();
  const int64_t vocab = a[4] == Py_None ? (g.next(), stride) : g.i64();
  void* s = g.stream();
  if (!g.ok || vocab != (int32_t)vocab) Py_RETURN_NONE;
  PTD_CALL(p_ptd_topk_draft(logits, dt, rows, (int32_t)vocab, stride, k, idx, val, s));
}

// (tree, tokens, target, target_stride, accepted, accept_len, bonus, dev_status, stream)
PyObject* verify_greedy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 9);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const int32_t* tokens = g.i32();
  const int32_t* target = g.i32();
  const int32_t stride = g.num();
  int32_t* acc = g.i32();
  int32_t* len = g.i32();
  int32_t* bonus = g.i32();
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_verify_greedy(tree, tokens, target, stride, acc, len, bonus, status, s));
}

// (tree, cache, accepted, accept_len, new_ctx, stream)
PyObject* kv_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 6);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  const int32_t* acc = g.i32();
  const int32_t* len = g.i32();
  int32_t* ctx = g.i32();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_kv_compact(tree, cache, acc, len, ctx, s));
}

// (tree, tokens, logits, temperature, u_accept, u_bonus, accepted, accept_len, bonus, dev_status, stream)
PyObject* verify_sampling(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 11);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const int32_t* tokens = g.i32();
  PyObject* lg = g.next();
  const ptd_dtype dt = g.kind(lg);
  int64_t rows, vocab, stride;
  const void* logits = g.rows2(lg, dt == PTD_BF16 ? g_bf16 : g_f32, &rows, &vocab, &stride);
  const float temperature = g.real();
  const float* ua = g.f32();
  const float* ub = g.f32();
  int32_t* acc = g.i32();
  int32_t* len = g.i32();
  int32_t* bonus = g.i32();
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok || vocab != (int32_t)vocab) Py_RETURN_NONE;
  PTD_CALL(p_ptd_verify_sampling(tree, tokens, logits, dt, (int32_t)vocab, stride, temperature, ua, ub, acc, len,
                                    bonus, status, s));
}

// (tree, cache, tokens, target, target_stride, accepted, accept_len, bonus, new_ctx, dev_status, stream)
PyObject* verify_and_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 11);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  const int32_t* tokens = g.i32();
  const int32_t* target = g.i32();
  const int32_t stride = g.num();
  int32_t* acc = g.i32();
  int32_t* len = g.i32();
  int32_t* bonus = g.i32();
  int32_t* ctx = g.i32();
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_verify_and_compact(tree, cache, tokens, target, stride, acc, len, bonus, ctx, status, s));
}

// (tree, cache, bufs, stream)
PyObject* tree_verify_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 4);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  const ptd_step_args* args = g.structure<ptd_step_args>();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_tree_verify_step(tree, cache, args, s));
}

// (in_count, in_parents, in_tokens, drafts, expand, width, max_depth, capacity, out_count, out_parents,
//  out_tokens, out_depths, old_to_new, dev_status, stream)
PyObject* draft_tree_update(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 15);
  if (!g.ok) Py_RETURN_NONE;
  int64_t B, stride, d0, d1, rows, dstride;
  const int32_t* in_count = g.i32();
  g.dims2(a[1], &B, &stride);
  const int32_t* in_parents = g.i32();
  g.dims2(a[2], &d0, &d1);
  if (d0 != B || d1 != stride) g.ok = false;
  const int32_t* in_tokens = g.i32();
  g.dims2(a[3], &rows, &dstride);
  if (rows != B * stride) g.ok = false;
  const int32_t* drafts = g.i32();
  const int32_t expand = g.num(), width = g.num(), max_depth = g.num(), capacity = g.num();
  int32_t* out_count = g.i32();
  int32_t* out[3];
  for (int32_t*& o : out) {
    g.dims2(a[g.i], &d0, &d1);
    if (d0 != B || d1 != capacity) g.ok = false;
    o = g.i32();
  }
  g.dims2(a[12], &d0, &d1);
  if (d0 != B || d1 != stride) g.ok = false;
  int32_t* old_to_new = g.i32();
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok || B != (int32_t)B || stride != (int32_t)stride || dstride != (int32_t)dstride) Py_RETURN_NONE;
  PTD_CALL(p_ptd_draft_tree_update((int32_t)B, (int32_t)stride, in_count, in_parents, in_tokens, drafts,
                                      (int32_t)dstride, expand, width, max_depth, capacity, out_count, out[0], out[1],
                                      out[2], old_to_new, status, s));
}

// (pool buffer, capacity, max_load, step, count, parents, tokens, dev_status, stream)
PyObject* pool_merge(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 9);
  if (!g.ok) Py_RETURN_NONE;
  void* pool = g.tensor();
  const int32_t capacity = g.num(), max_load = g.num(), step = g.num();
  const int32_t* count = g.i32();
  const int32_t* parents = g.i32();
  const int32_t* tokens = g.i32();
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_pool_merge(pool, capacity, max_load, step, count, parents, tokens, status, s));
}

// (pool buffer, capacity, root_token, width, max_depth, max_nodes, out_count, out_parents, out_tokens, stream)
PyObject* pool_retrieve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 10);
  if (!g.ok) Py_RETURN_NONE;
  const void* pool = g.tensor();
  const int32_t capacity = g.num();
  const int32_t* root = g.i32();
  const int32_t width = g.num(), max_depth = g.num(), max_nodes = g.num();
  int32_t* count = g.i32();
  int32_t* out[2];
  for (int32_t*& o : out) {
    PyObject* t = a[g.i];
    o = g.i32();
    if (!g.ok) Py_RETURN_NONE;
    if (look::nbytes(t) < 4 * (int64_t)max_nodes) g.fail();
  }
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_pool_retrieve(pool, capacity, root, width, max_depth, max_nodes, count, out[0], out[1], s));
}

// (tree, cache, layer_begin, num_layers, q, num_q_heads, k, v, rope_base, positions_out, dev_status, stream)
PyObject* tree_rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 12);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (!g.ok) Py_RETURN_NONE;
  PyObject* dt = cache->dtype == PTD_BF16 ? g_bf16 : g_f32;
  const int32_t l0 = g.num(), nl = g.num();
  void* q = g.tensor(dt);
  const int32_t hq = g.num();
  const void* k = g.tensor(dt);
  const void* v = g.tensor(dt);
  const float base = g.real();
  int32_t* pos = a[9] == Py_None ? (g.next(), nullptr) : g.i32();
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_tree_rope_append(tree, cache, l0, nl, q, hq, k, v, base, pos, status, s));
}

// (hidden, weight, k, out_idx, out_val, workspace, dev_status, stream)
PyObject* lm_head_topk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 8);
  if (!g.ok) Py_RETURN_NONE;
  int64_t rows, d, hstride, vocab, wd, wstride;
  const void* hidden = g.rows2(g.next(), g_bf16, &rows, &d, &hstride);
  if (!g.ok) Py_RETURN_NONE;
  const void* weight = g.rows2(g.next(), g_bf16, &vocab, &wd, &wstride);
  const int32_t k = g.num();
  int32_t* idx = g.i32();
  float* val = g.f32();
  size_t wsb;
  if (a[g.i] == Py_None) Py_RETURN_NONE;
  void* ws = g.optional(&wsb);
  int32_t* status = g.i32();
  void* s = g.stream();
  if (!g.ok || d != wd || rows != (int32_t)rows || vocab != (int32_t)vocab || d != (int32_t)d) Py_RETURN_NONE;
  PTD_CALL(p_ptd_lm_head_topk(hidden, (int32_t)rows, hstride, weight, (int32_t)vocab, wstride, (int32_t)d, k, idx,
                                 val, ws, wsb, status, s));
}

// (prompt, cache, pages, slots, positions, dev_status, stream)
PyObject* prompt_slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 7);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_prompt* prompt = g.structure<ptd_prompt>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (g.ok) g.batch_of(a[1], prompt, cache);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_page_pool* held = a[2] == Py_None ? (g.next(), nullptr) : g.structure<ptd_page_pool>();
  if (!g.ok) Py_RETURN_NONE;
  ptd_page_pool pool = {};
  if (held != nullptr) {   // sizes: (sequences, pages, device) of the pool's tensors
    PyObject* sizes = PyObject_GetAttr(a[2], s_sizes);
    PyObject* table = PyObject_GetAttr(a[1], s_block_table);
    int64_t rows = 0, cols = 0;
    if (sizes == nullptr || table == nullptr || table == Py_None || !PyTuple_CheckExact(sizes) || PyTuple_GET_SIZE(sizes) != 3 ||
        PyLong_AsLongLong(PyTuple_GET_ITEM(sizes, 0)) != prompt->batch ||
        PyLong_AsLongLong(PyTuple_GET_ITEM(sizes, 1)) != cache->num_pages) {
      g.fail();
    } else {
      g.device = PyLong_AsLongLong(PyTuple_GET_ITEM(sizes, 2));
      g.dims2(table, &rows, &cols);
      if (rows != prompt->batch) g.ok = false;
    }
    Py_XDECREF(sizes);
    Py_XDECREF(table);
    pool = *held;
    pool.block_table = const_cast<int32_t*>(cache->block_table);
  }
  int32_t* slots = g.i32_of(prompt->total_tokens);
  int32_t* positions = g.i32_of(prompt->total_tokens);
  g.on(a[5]);
  int32_t* status = g.i32();
  g.on_attr(a[0], s_ctx_lens);
  g.on_attr(a[1], s_k);
  g.on_current();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_prompt_slots(prompt, cache, held != nullptr ? &pool : nullptr, slots, positions, status, s));
}

// (prompt, cache, layer, slots, positions, q, k, v, q_out, rope_base, dev_status, stream)
PyObject* prompt_rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 12);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_prompt* prompt = g.structure<ptd_prompt>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (g.ok) g.batch_of(a[1], prompt, cache);
  if (!g.ok) Py_RETURN_NONE;
  PyObject* dt = cache->dtype == PTD_BF16 ? g_bf16 : g_f32;
  const int32_t layer = g.num();
  const int32_t* slots = g.i32_of(prompt->total_tokens);
  const int32_t* positions = g.i32_of(prompt->total_tokens);
  int64_t hq = 0, hkv = cache->num_kv_heads, qs, ks, vs, os;
  const void* q = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hq, &qs);
  const void* k = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hkv, &ks);
  const void* v = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hkv, &vs);
  void* out = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hq, &os);
  const float base = g.real();
  g.on(a[10]);
  int32_t* status = g.i32();
  g.on_attr(a[1], s_k);
  g.on_current();
  void* s = g.stream();
  if (!g.ok || hq != (int32_t)hq) Py_RETURN_NONE;
  PTD_CALL(p_ptd_prompt_rope_append(prompt, cache, layer, slots, positions, q, qs, (int32_t)hq, k, ks, v, vs, base, out, os,
                                    status, s));
}

// (prompt, cache, layer, q, out, dev_status, scale, workspace, stream)
PyObject* prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 9);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_prompt* prompt = g.structure<ptd_prompt>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (g.ok) g.batch_of(a[1], prompt, cache);
  if (!g.ok) Py_RETURN_NONE;
  PyObject* dt = cache->dtype == PTD_BF16 ? g_bf16 : g_f32;
  const int32_t layer = g.num();
  int64_t hq = 0, qs, os = 0;
  const void* q = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hq, &qs);
  void* out = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hq, &os);
  if (os != hq * cache->head_dim && prompt->total_tokens > 1) g.ok = false;   // out is contiguous
  g.on(a[5]);
  int32_t* status = g.i32();
  const float scale = g.real();
  size_t wsb;
  if (a[7] != Py_None) g.on(a[7]);
  void* ws = g.optional(&wsb);
  g.on_attr(a[0], s_ctx_lens);
  g.on_attr(a[1], s_k);
  g.on_current();
  void* s = g.stream();
  if (!g.ok || hq != (int32_t)hq) Py_RETURN_NONE;
  PTD_CALL(p_ptd_prompt_attention(prompt, cache, layer, q, qs, (int32_t)hq, scale, out, ws, wsb, status, s));
}

// (prompt, cache, layer, slots, positions, q, k, v, q_out, q_weight, k_weight, eps, rope_base, dev_status, stream)
PyObject* prompt_norm_rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 15);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_prompt* prompt = g.structure<ptd_prompt>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (g.ok) g.batch_of(a[1], prompt, cache);
  if (!g.ok) Py_RETURN_NONE;
  PyObject* dt = cache->dtype == PTD_BF16 ? g_bf16 : g_f32;
  const int32_t layer = g.num();
  const int32_t* slots = g.i32_of(prompt->total_tokens);
  const int32_t* positions = g.i32_of(prompt->total_tokens);
  int64_t hq = 0, hkv = cache->num_kv_heads, qs, ks, vs, os;
  const void* q = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hq, &qs);
  const void* k = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hkv, &ks);
  const void* v = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hkv, &vs);
  void* out = g.rows3(dt, prompt->total_tokens, cache->head_dim, &hq, &os);
  const int64_t want[1] = {cache->head_dim};
  const void* qw = g.shaped(dt, 1, want);
  const void* kw = g.shaped(dt, 1, want);
  const float eps = g.real(), base = g.real();
  int32_t* status = static_cast<int32_t*>(g.tensor_on(g.next(), g_i32));
  g.on_attr(a[1], s_k);
  g.on_current();
  void* s = g.stream();
  if (!g.ok || hq != (int32_t)hq) Py_RETURN_NONE;
  PTD_CALL(p_ptd_prompt_norm_rope_append(prompt, cache, layer, slots, positions, q, qs, (int32_t)hq, k, ks, v, vs, qw, kw, eps,
                                         base, out, os, status, s));
}

// (tree, cache, layer_begin, q, k, v, q_out, q_weight, k_weight, eps, rope_base, dev_status, positions_out, stream)
PyObject* tree_norm_rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 14);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_tree* tree = g.structure<ptd_tree>();
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  if (!g.ok) Py_RETURN_NONE;
  PyObject* dt = cache->dtype == PTD_BF16 ? g_bf16 : g_f32;
  const int32_t l0 = g.num();
  if ((PyObject*)Py_TYPE(a[3]) != g_tensor) Py_RETURN_NONE;
  int64_t d[4];
  if (g.dims(a[3], d) != 4) Py_RETURN_NONE;
  const int64_t q_shape[4] = {d[0], tree->total_nodes, d[2], cache->head_dim};
  const int64_t kv_shape[4] = {d[0], tree->total_nodes, cache->num_kv_heads, cache->head_dim}, w_shape[2] = {d[0], cache->head_dim};
  const void* q = g.shaped(dt, 4, q_shape);
  const void* k = g.shaped(dt, 4, kv_shape);
  const void* v = g.shaped(dt, 4, kv_shape);
  void* out = g.shaped(dt, 4, q_shape);
  const void* qw = g.shaped(dt, 2, w_shape);
  const void* kw = g.shaped(dt, 2, w_shape);
  const float eps = g.real(), base = g.real();
  int32_t* status = static_cast<int32_t*>(g.tensor_on(g.next(), g_i32));
  int32_t* pos = a[12] == Py_None ? (g.next(), nullptr) : g.i32_of(tree->total_nodes);
  g.on_attr(a[0], s_ctx_lens);
  g.on_attr(a[1], s_k);
  g.on_current();
  void* s = g.stream();
  if (!g.ok || d[0] != (int32_t)d[0] || d[2] != (int32_t)d[2]) Py_RETURN_NONE;
  PTD_CALL(p_ptd_tree_norm_rope_append(tree, cache, l0, (int32_t)d[0], q, (int32_t)d[2], k, v, qw, kw, eps, base, out, pos,
                                       status, s));
}

// (logits, tokens, out_logprob, out_entropy, out_idx, out_val, dev_status, temperature, stream)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 9);
  if (!g.ok) Py_RETURN_NONE;
  PyObject* lg = g.next();
  const ptd_dtype dt = g.kind(lg);
  int64_t rows, vocab, stride;
  const void* logits = g.rows2(lg, dt == PTD_BF16 ? g_bf16 : g_f32, &rows, &vocab, &stride);
  g.on(lg);
  if (!g.ok) Py_RETURN_NONE;
  const Args::Logprobs x = g.logprobs(rows);
  int32_t* status = static_cast<int32_t*>(g.tensor_on(g.next(), g_i32));
  const float temperature = g.real();
  g.on_current();
  void* s = g.stream();
  if (!g.ok || vocab != (int32_t)vocab) Py_RETURN_NONE;
  PTD_CALL(p_ptd_token_logprobs(logits, dt, rows, (int32_t)vocab, stride, x.tokens, temperature, x.k, x.logprob, x.entropy, x.idx,
                                x.val, status, s));
}

// (hidden, weight, tokens, out_logprob, out_entropy, out_idx, out_val, workspace, dev_status, temperature, stream)
PyObject* lm_head_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 11);
  if (!g.ok) Py_RETURN_NONE;
  int64_t rows, d, hstride, vocab, wd, wstride;
  const void* hidden = g.rows2(g.next(), g_bf16, &rows, &d, &hstride);
  if (!g.ok) Py_RETURN_NONE;
  const void* weight = g.rows2(g.next(), g_bf16, &vocab, &wd, &wstride);
  g.on(a[0]);
  g.on(a[1]);
  if (!g.ok) Py_RETURN_NONE;
  const Args::Logprobs x = g.logprobs(rows);
  size_t wsb;
  if (a[7] == Py_None) Py_RETURN_NONE;
  g.on(a[7]);
  void* ws = g.optional(&wsb);
  int32_t* status = static_cast<int32_t*>(g.tensor_on(g.next(), g_i32));
  const float temperature = g.real();
  g.on_current();
  void* s = g.stream();
  if (!g.ok || d != wd || rows != (int32_t)rows || vocab != (int32_t)vocab || d != (int32_t)d) Py_RETURN_NONE;
  PTD_CALL(p_ptd_lm_head_logprobs(hidden, (int32_t)rows, hstride, weight, (int32_t)vocab, wstride, (int32_t)d, x.tokens,
                                  temperature, x.k, x.logprob, x.entropy, x.idx, x.val, ws, wsb, status, s));
}

// (cache, source, target, parents, lens, workspace, dev_status, stream)
PyObject* page_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g(a, n, 8);
  if (!g.ok) Py_RETURN_NONE;
  const ptd_kv_cache* cache = g.structure<ptd_kv_cache>();
  const ptd_page_set* from = g.structure<ptd_page_set>();
  const ptd_page_set* to = g.structure<ptd_page_set>();
  if (!g.ok) Py_RETURN_NONE;
  for (int i = 1; i <= 2; ++i) {   // sizes: (entries of a row, pages, device) of the set's tensors
    PyObject* sizes = PyObject_GetAttr(a[i], s_sizes);
    if (sizes == nullptr || !PyTuple_CheckExact(sizes) || PyTuple_GET_SIZE(sizes) != 3 ||
        PyLong_AsLongLong(PyTuple_GET_ITEM(sizes, 0)) != cache->max_pages ||
        PyLong_AsLongLong(PyTuple_GET_ITEM(sizes, 1)) != cache->num_pages) {
      g.fail();
    } else {
      const int64_t on = PyLong_AsLongLong(PyTuple_GET_ITEM(sizes, 2));
      if (g.device >= 0 && g.device != on) g.ok = false;
      g.device = on;
    }
    Py_XDECREF(sizes);
  }
  const int32_t* parents = g.i32_of(to->batch);
  const int32_t* lens = g.i32_of(to->batch);
  size_t wsb;
  if (a[5] == Py_None) Py_RETURN_NONE;
  g.on(a[5]);
  void* ws = g.optional(&wsb);
  int32_t* status = static_cast<int32_t*>(g.tensor_on(g.next(), g_i32));
  g.on_attr(a[0], s_k);
  g.on_current();
  void* s = g.stream();
  if (!g.ok) Py_RETURN_NONE;
  PTD_CALL(p_ptd_page_fork(cache, from, to, parents, lens, ws, wsb, status, s));
}

// Whether the process's torch is the version that the tensors' layout was compiled from (else a Python error).
bool same_torch() {
  PyObject* torch = PyImport_ImportModule("torch");
  PyObject* version = torch != nullptr ? PyObject_GetAttrString(torch, "__version__") : nullptr;
  const char* here = version != nullptr ? PyUnicode_AsUTF8(version) : nullptr;
  const bool same = here != nullptr && strcmp(here, PTD_TORCH_VERSION) == 0;
  if (!same && !PyErr_Occurred())
    PyErr_Format(PyExc_RuntimeError, "_ptdcall.so was compiled for torch " PTD_TORCH_VERSION ", this is %s: run __graft_entry__.build()",
                 here);
  Py_XDECREF(version);
  Py_XDECREF(torch);
  return same;
}

// load(path of libptd.so, Tensor type, int32, float32, bfloat16, raw stream getter, device getter)
PyObject* load(PyObject*, PyObject* args) {
  const char* path;
  PyObject* o[6];
  if (!PyArg_ParseTuple(args, "sOOOOOO", &path, &o[0], &o[1], &o[2], &o[3], &o[4], &o[5])) return nullptr;
  if (!same_torch()) return nullptr;
  void* h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
  if (h == nullptr) {
    PyErr_SetString(PyExc_RuntimeError, dlerror());
    return nullptr;
  }
#define PTD_RESOLVE(f)                                                      \
  p_##f = reinterpret_cast<decltype(&f)>(dlsym(h, #f));                     \
  if (p_##f == nullptr) {                                                   \
    PyErr_SetString(PyExc_RuntimeError, "libptd.so has no symbol " #f);     \
    return nullptr;                                                         \
  }
  PTD_FUNCTIONS(PTD_RESOLVE)
#undef PTD_RESOLVE
  for (PyObject* x : o) Py_INCREF(x);
  g_direct = o[0] == THPVariableClass;
  g_tensor = o[0], g_i32 = o[1], g_f32 = o[2], g_bf16 = o[3], g_raw_stream = o[4], g_get_device = o[5];
  Py_RETURN_NONE;
}

#define PTD_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PTD_METHOD(tree_attention),
                         PTD_METHOD(topk_draft),
                         PTD_METHOD(verify_greedy),
                         PTD_METHOD(kv_compact),
                         PTD_METHOD(verify_sampling),
                         PTD_METHOD(verify_and_compact),
                         PTD_METHOD(tree_verify_step),
                         PTD_METHOD(draft_tree_update),
                         PTD_METHOD(pool_merge),
                         PTD_METHOD(pool_retrieve),
                         PTD_METHOD(tree_rope_append),
                         PTD_METHOD(lm_head_topk),
                         PTD_METHOD(prompt_slots),
                         PTD_METHOD(prompt_rope_append),
                         PTD_METHOD(prompt_attention),
                         PTD_METHOD(prompt_norm_rope_append),
                         PTD_METHOD(tree_norm_rope_append),
                         PTD_METHOD(token_logprobs),
                         PTD_METHOD(lm_head_logprobs),
                         PTD_METHOD(page_fork),
                         {"load", load, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ptdcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ptdcall(void) {
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_nbytes = PyUnicode_InternFromString("nbytes");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_c = PyUnicode_InternFromString("c");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_k = PyUnicode_InternFromString("k");
  s_block_table = PyUnicode_InternFromString("block_table");
  s_ctx_lens = PyUnicode_InternFromString("ctx_lens");
  s_sizes = PyUnicode_InternFromString("sizes");
  return PyModule_Create(&module);
}
