// The binding's calls of the grouped-query part: checks of torch tensors and their way into the C ABI.  (Read attribute by attribute in
// Python, the 8 to 11 tensors of a call cost 4 us, more than the call itself and twice what a step's tables take on the GPU; here 0.2.)
// A module of its own beside the library, which knows nothing of Python; it gets the library's functions by address.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <limits>
#include <string>

#include "../../include/omniattn.h"

namespace {

PyObject *g_error, *g_device, *g_stream;  // OmniAttnError, and torch's functions for the current device and a device's current stream
PyObject* s_cuda_stream;
decltype(&omniattn_table_extend) g_extend;
decltype(&omniattn_table_release) g_release;
decltype(&omniattn_gqa_append) g_append;
decltype(&omniattn_gqa_decode) g_decode;
decltype(&omniattn_table_truncate) g_truncate;
decltype(&omniattn_tree_masks) g_tree_masks;
decltype(&omniattn_gqa_tree) g_tree;
decltype(&omniattn_tree_verify) g_verify;
decltype(&omniattn_gqa_keep) g_keep;

struct Refused {};  // a Python error is set

[[noreturn]] void refuse(const std::string& what) {
  if (PyObject* e = PyObject_CallFunction(g_error, "is", OMNIATTN_EINVAL, what.c_str())) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Refused();
}

// The tensors of a call, all on one device.
struct Call {
  int device = -1;

  const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor wanted");
    return THPVariable_Unpack(o);
  }
  bool here(const at::Tensor& t) {
    if (!t.is_cuda()) return false;
    if (device < 0) device = t.get_device();
    return t.get_device() == device;
  }
  int32_t* ints(const at::Tensor& t, int64_t n, const char* name) {
    if (t.scalar_type() != at::kInt || t.numel() != n || !t.is_contiguous() || !here(t))
      refuse(std::string(name) + ": int32 CUDA tensor of " + std::to_string(n) + " elements wanted");
    return static_cast<int32_t*>(t.data_ptr());
  }
  int32_t* ints(PyObject* o, int64_t n, const char* name) { return ints(tensor(o, name), n, name); }
  const int32_t* ints_or_none(PyObject* o, int64_t n, const char* name) { return o == Py_None ? nullptr : ints(o, n, name); }
  float* floats(PyObject* o, int64_t n, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != at::kFloat || t.numel() != n || !t.is_contiguous() || !here(t))
      refuse(std::string(name) + ": contiguous fp32 CUDA tensor of " + std::to_string(n) + " elements wanted");
    return static_cast<float*>(t.data_ptr());
  }
  uint64_t* masks(PyObject* o, int64_t n) {
    const at::Tensor& t = tensor(o, "masks");
    if (t.scalar_type() != at::kLong || t.numel() != n || !t.is_contiguous() || !here(t)) refuse("masks: int64 CUDA tensor of " + std::to_string(n) + " elements wanted");
    return static_cast<uint64_t*>(t.data_ptr());
  }
  // rows of a matrix with any stride from row to row
  void* matrix(const at::Tensor& t, int64_t rows, int64_t columns, const char* name, int64_t& stride) {
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != columns || (t.stride(1) != 1 && columns > 1) || !here(t))
      refuse(std::string(name) + ": CUDA tensor [" + std::to_string(rows) + ", " + std::to_string(columns) + "] wanted, its rows contiguous");
    stride = rows > 1 ? t.stride(0) : columns;
    return t.data_ptr();
  }
  void* workspace(PyObject* o, size_t& bytes) {
    bytes = 0;
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, "workspace");
    if (!t.is_contiguous() || !here(t)) refuse("workspace: contiguous CUDA tensor wanted");
    bytes = t.nbytes();
    return t.data_ptr();
  }
  int32_t* table(PyObject* o, int64_t batch, int32_t& columns, int64_t& stride) {
    const at::Tensor& t = tensor(o, "page_table");
    if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != batch || (t.stride(1) != 1 && t.size(1) > 1) || t.size(1) > INT32_MAX || !here(t))
      refuse("page_table: int32 CUDA tensor [batch, pages] wanted, its rows contiguous");
    columns = static_cast<int32_t>(t.size(1));
    stride = t.size(0) > 1 ? t.stride(0) : columns;  // (of a single row it may be anything)
    return static_cast<int32_t*>(t.data_ptr());
  }
  // bf16 rows [tokens, heads, dim] with any stride from token to token
  void* rows(const at::Tensor& t, int64_t heads, int64_t dim, const char* name, int64_t& stride) {
    if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || t.size(1) != heads || t.size(2) != dim || t.stride(2) != 1 || (t.stride(1) != dim && heads != 1) ||
        t.size(0) > INT32_MAX || !here(t))
      refuse(std::string(name) + ": bf16 CUDA tensor [tokens, " + std::to_string(heads) + ", " + std::to_string(dim) + "] wanted, a token's rows contiguous");
    stride = t.size(0) > 1 ? t.stride(0) : heads * dim;
    return t.data_ptr();
  }
  void* stream(PyObject* given) {
    PyObject* x;
    if (given != Py_None) {
      x = PyObject_GetAttr(given, s_cuda_stream);
    } else {
      PyObject* current = PyObject_CallNoArgs(g_device);
      if (!current) throw Refused();
      const bool same = PyLong_AsLong(current) == device;
      x = same ? PyObject_CallOneArg(g_stream, current) : nullptr;
      Py_DECREF(current);
      if (!same) refuse("tensors on the current device wanted");
    }
    if (!x) throw Refused();
    void* handle = PyLong_AsVoidPtr(x);
    Py_DECREF(x);
    if (!handle && PyErr_Occurred()) throw Refused();
    return handle;
  }
};

int32_t small(int64_t n, const char* name) {
  if (n > INT32_MAX) refuse(std::string(name) + ": too many");
  return static_cast<int32_t>(n);
}
int32_t index(PyObject* o, const char* name) {
  PyObject* i = PyNumber_Index(o);
  if (!i) throw Refused();
  const long long x = PyLong_AsLongLong(i);
  Py_DECREF(i);
  if (PyErr_Occurred() || x < INT32_MIN || x > INT32_MAX) {
    PyErr_Clear();
    refuse(std::string(name) + ": a number of 32 bits wanted");
  }
  return static_cast<int32_t>(x);
}

// A layer's cache; or several layers', one behind the other, where the call takes them (layers not null).
struct Cache {
  void *k, *v;
  float *k_scales, *v_scales;
};
Cache cache_of(Call& call, PyObject* const* a, omniattn_gqa_t& g, int32_t* layers = nullptr) {
  const at::Tensor &k = call.tensor(a[0], "k_cache"), &v = call.tensor(a[1], "v_cache"), &ks = call.tensor(a[2], "k_scales"), &vs = call.tensor(a[3], "v_scales");
  if (k.scalar_type() != at::kFloat8_e4m3fn || v.scalar_type() != at::kFloat8_e4m3fn || ks.scalar_type() != at::kFloat || vs.scalar_type() != at::kFloat ||
      (k.dim() != 4 && !(layers && k.dim() == 5)) || ks.dim() != k.dim() - 1 || v.sizes() != k.sizes() || vs.sizes() != ks.sizes())
    refuse("cache (float8_e4m3fn) [pages, KV heads, 128, head width] with scales (float32) [pages, KV heads, 128 / tokens] wanted, for K and V alike");
  if (!k.is_contiguous() || !v.is_contiguous() || !ks.is_contiguous() || !vs.is_contiguous() || !call.here(k) || !call.here(v) || !call.here(ks) || !call.here(vs))
    refuse("cache and scales: contiguous CUDA tensors wanted");
  const int64_t at = k.dim() - 4;  // dimensions in front of a layer's
  if (ks.size(0) != k.size(0) || ks.size(at) != k.size(at) || ks.size(at + 1) != k.size(at + 1) || ks.size(at + 2) <= 0 || k.size(at + 2) % ks.size(at + 2) != 0)
    refuse("scales: for every page and KV head of the cache wanted, their number a divisor of a page's tokens");
  if (layers) *layers = at ? small(k.size(0), "layers") : 1;
  g.num_pages = k.size(at);
  g.num_kv_heads = small(k.size(at + 1), "KV heads");
  g.page_size = small(k.size(at + 2), "tokens of a page");
  g.head_dim = small(k.size(at + 3), "head width");
  g.scale_tokens = g.page_size / static_cast<int32_t>(ks.size(at + 2));
  return Cache{k.data_ptr(), v.data_ptr(), static_cast<float*>(ks.data_ptr()), static_cast<float*>(vs.data_ptr())};
}

// (f calls the library and nothing else: it may not throw)
template <typename F>
int without_gil(F f) {
  PyThreadState* state = PyEval_SaveThread();
  const int rc = f();
  PyEval_RestoreThread(state);
  return rc;
}

// seq_lens, new_lens, free_pages, free_count, page_table, seq_lens_out, free_count_out, q_start, slot_map, stream
int extend(PyObject* const* a) {
  Call c;
  omniattn_table_t t{};
  const at::Tensor &lens = c.tensor(a[0], "seq_lens"), &free_pages = c.tensor(a[2], "free_pages"), &slots = c.tensor(a[8], "slot_map");
  const int64_t batch = lens.numel();
  t.batch = small(batch, "requests");
  t.page_size = OMNIATTN_PAGE;
  t.max_tokens = small(slots.numel(), "tokens");
  t.num_pages = free_pages.numel();
  int32_t *seq_lens = c.ints(lens, batch, "seq_lens"), *new_lens = c.ints(a[1], batch, "new_lens"), *free_at = c.ints(free_pages, t.num_pages, "free_pages"),
          *count = c.ints(a[3], 1, "free_count"), *table = c.table(a[4], batch, t.max_pages_per_seq, t.page_table_stride),
          *lens_out = c.ints(a[5], batch, "seq_lens_out"), *count_out = c.ints(a[6], 1, "free_count_out"), *q_start = c.ints(a[7], batch + 1, "q_start"),
          *slot_map = c.ints(slots, t.max_tokens, "slot_map");
  void* const stream = c.stream(a[9]);
  return without_gil([&] { return g_extend(&t, seq_lens, new_lens, free_at, count, table, lens_out, count_out, q_start, slot_map, stream); });
}

// seq_lens, done, page_table, free_pages, free_count, stream
int release(PyObject* const* a) {
  Call c;
  omniattn_table_t t{};
  const at::Tensor &lens = c.tensor(a[0], "seq_lens"), &pages = c.tensor(a[3], "free_pages");
  const int64_t batch = lens.numel();
  t.batch = small(batch, "requests");
  t.page_size = OMNIATTN_PAGE;
  t.num_pages = pages.numel();
  int32_t *seq_lens = c.ints(lens, batch, "seq_lens"), *done = c.ints(a[1], batch, "done"), *table = c.table(a[2], batch, t.max_pages_per_seq, t.page_table_stride),
          *free_at = c.ints(pages, t.num_pages, "free_pages"), *count = c.ints(a[4], 1, "free_count");
  void* const stream = c.stream(a[5]);
  return without_gil([&] { return g_release(&t, done, seq_lens, table, free_at, count, stream); });
}

// k_new, v_new, slot_map, k_cache, v_cache, k_scales, v_scales, stream
int append(PyObject* const* a) {
  Call c;
  omniattn_gqa_t g{};
  const Cache cache = cache_of(c, a + 3, g);
  g.batch = g.max_pages_per_seq = 1;
  g.page_table_stride = 1;
  g.num_q_heads = g.num_kv_heads;
  g.softmax_scale = 1.f;
  const at::Tensor &k_new = c.tensor(a[0], "k_new"), &v_new = c.tensor(a[1], "v_new");
  int64_t k_stride, v_stride;
  const void *k = c.rows(k_new, g.num_kv_heads, g.head_dim, "k_new", k_stride), *v = c.rows(v_new, g.num_kv_heads, g.head_dim, "v_new", v_stride);
  if (k_new.size(0) != v_new.size(0)) refuse("k_new and v_new: as many tokens wanted");
  const int32_t n = static_cast<int32_t>(k_new.size(0));
  const int32_t* slots = c.ints(a[2], n, "slot_map");
  void* const stream = c.stream(a[7]);
  return without_gil([&] { return g_append(&g, n, k, k_stride, v, v_stride, slots, cache.k, cache.v, cache.k_scales, cache.v_scales, stream); });
}

// q, k_cache, v_cache, k_scales, v_scales, page_table, seq_lens, q_start, [of a tree: masks,] out, lse, workspace, sink, window, softmax_scale, stream
template <bool TREE>
int attend(PyObject* const* a) {
  Call c;
  omniattn_gqa_t g{};
  const Cache cache = cache_of(c, a + 1, g);
  const at::Tensor &q = c.tensor(a[0], "q"), &lens = c.tensor(a[6], "seq_lens"), &out = c.tensor(a[8 + TREE], "out"), &lse = c.tensor(a[9 + TREE], "lse");
  const int64_t batch = lens.numel(), heads = q.dim() == 3 ? q.size(1) : 0;
  int64_t q_stride;
  const void* rows = c.rows(q, heads, g.head_dim, "q", q_stride);
  g.batch = small(batch, "requests");
  g.num_queries = static_cast<int32_t>(q.size(0));
  g.num_q_heads = small(heads, "query heads");
  const int32_t* table = c.table(a[5], batch, g.max_pages_per_seq, g.page_table_stride);
  const int32_t* seq_lens = c.ints(lens, batch, "seq_lens");
  const int32_t* q_start = c.ints_or_none(a[7], batch + 1, "q_start");
  const uint64_t* masks = TREE ? c.masks(a[8], g.num_queries) : nullptr;
  const bool fp32 = out.scalar_type() == at::kFloat;
  if ((!fp32 && out.scalar_type() != at::kBFloat16) || out.sizes() != q.sizes() || !out.is_contiguous() || !c.here(out))
    refuse("out: contiguous bf16 or fp32 CUDA tensor shaped like q wanted");
  if (lse.scalar_type() != at::kFloat || lse.dim() != 2 || lse.size(0) != q.size(0) || lse.size(1) != heads || !lse.is_contiguous() || !c.here(lse))
    refuse("lse: contiguous fp32 CUDA tensor [tokens, query heads] wanted");
  size_t bytes;
  void* const workspace = c.workspace(a[10 + TREE], bytes);
  g.sink = index(a[11 + TREE], "sink");
  g.window = index(a[12 + TREE], "window");
  const double scale = PyFloat_AsDouble(a[13 + TREE]);
  if (scale == -1.0 && PyErr_Occurred()) throw Refused();
  g.softmax_scale = static_cast<float>(scale);
  g.out_dtype = fp32 ? OMNIATTN_FP32 : OMNIATTN_BF16;
  void *const stream = c.stream(a[14 + TREE]), *const result = out.data_ptr();
  float* const sums = static_cast<float*>(lse.data_ptr());
  return without_gil([&] {
    if constexpr (TREE)
      return g_tree(&g, rows, q_stride, cache.k, cache.v, cache.k_scales, cache.v_scales, table, seq_lens, q_start, masks, result, sums, workspace, bytes, stream);
    return g_decode(&g, rows, q_stride, cache.k, cache.v, cache.k_scales, cache.v_scales, table, seq_lens, q_start, result, sums, workspace, bytes, stream);
  });
}

int decode(PyObject* const* a) { return attend<false>(a); }
int tree(PyObject* const* a) { return attend<true>(a); }

// seq_lens, dropped, page_table, free_pages, free_count, seq_lens_out, free_count_out, stream
int truncate(PyObject* const* a) {
  Call c;
  omniattn_table_t t{};
  const at::Tensor &lens = c.tensor(a[0], "seq_lens"), &pages = c.tensor(a[3], "free_pages");
  const int64_t batch = lens.numel();
  t.batch = small(batch, "requests");
  t.page_size = OMNIATTN_PAGE;
  t.num_pages = pages.numel();
  int32_t *seq_lens = c.ints(lens, batch, "seq_lens"), *dropped = c.ints(a[1], batch, "dropped"), *table = c.table(a[2], batch, t.max_pages_per_seq, t.page_table_stride),
          *free_at = c.ints(pages, t.num_pages, "free_pages"), *count = c.ints(a[4], 1, "free_count"), *lens_out = c.ints(a[5], batch, "seq_lens_out"),
          *count_out = c.ints(a[6], 1, "free_count_out");
  void* const stream = c.stream(a[7]);
  return without_gil([&] { return g_truncate(&t, seq_lens, dropped, table, free_at, count, lens_out, count_out, stream); });
}

// parents, seq_lens, q_start, masks, positions, stream
int tree_masks(PyObject* const* a) {
  Call c;
  const at::Tensor &parents = c.tensor(a[0], "parents"), &lens = c.tensor(a[1], "seq_lens");
  const int32_t batch = small(lens.numel(), "requests"), nodes = small(parents.numel(), "nodes");
  const int32_t *of = c.ints(parents, nodes, "parents"), *seq_lens = c.ints(lens, batch, "seq_lens"), *q_start = c.ints_or_none(a[2], (int64_t)batch + 1, "q_start");
  uint64_t* const masks = c.masks(a[3], nodes);
  int32_t* const positions = a[4] == Py_None ? nullptr : c.ints(a[4], nodes, "positions");
  void* const stream = c.stream(a[5]);
  return without_gil([&] { return g_tree_masks(batch, nodes, of, seq_lens, q_start, masks, positions, stream); });
}

// logits, draft_probs, tokens, parents, q_start, temperature, uniforms, path, out_tokens, logprobs, dropped, workspace, stream
int verify(PyObject* const* a) {
  Call c;
  omniattn_verify_t v{};
  const at::Tensor &logits = c.tensor(a[0], "logits"), &dropped = c.tensor(a[10], "dropped");
  const bool fp32 = logits.scalar_type() == at::kFloat;
  if ((!fp32 && logits.scalar_type() != at::kBFloat16) || logits.dim() != 2) refuse("logits: bf16 or fp32 CUDA tensor [nodes, vocabulary] wanted");
  const int64_t nodes = logits.size(0), vocab = logits.size(1), batch = dropped.numel();
  v.batch = small(batch, "requests");
  v.num_tokens = small(nodes, "nodes");
  v.vocab = small(vocab, "vocabulary");
  v.logits_dtype = fp32 ? OMNIATTN_FP32 : OMNIATTN_BF16;
  int64_t stride, draft_stride = 0;
  const void* const rows = c.matrix(logits, nodes, vocab, "logits", stride);
  const float* drafts = nullptr;
  if (a[1] != Py_None) {
    const at::Tensor& t = c.tensor(a[1], "draft_probs");
    if (t.scalar_type() != at::kFloat) refuse("draft_probs: fp32 wanted");
    drafts = static_cast<const float*>(c.matrix(t, nodes, vocab, "draft_probs", draft_stride));
  }
  const int32_t *tokens = c.ints(a[2], nodes, "tokens"), *parents = c.ints(a[3], nodes, "parents"), *q_start = c.ints_or_none(a[4], batch + 1, "q_start");
  const float *temperature = c.floats(a[5], batch, "temperature"), *uniforms = c.floats(a[6], 2 * nodes, "uniforms");
  int32_t *path = c.ints(a[7], nodes, "path"), *out = c.ints(a[8], nodes, "out_tokens"), *less = c.ints(dropped, batch, "dropped");
  float* const logprobs = a[9] == Py_None ? nullptr : c.floats(a[9], nodes, "logprobs");
  size_t bytes;
  void* const workspace = c.workspace(a[11], bytes);
  void* const stream = c.stream(a[12]);
  return without_gil([&] {
    return g_verify(&v, rows, stride, drafts, draft_stride, tokens, parents, q_start, temperature, uniforms, path, out, logprobs, less, workspace, bytes, stream);
  });
}

// path, seq_lens, q_start, page_table, k_cache, v_cache, k_scales, v_scales, stream
int keep(PyObject* const* a) {
  Call c;
  omniattn_gqa_t g{};
  int32_t layers;
  const Cache cache = cache_of(c, a + 4, g, &layers);
  const at::Tensor &way = c.tensor(a[0], "path"), &lens = c.tensor(a[1], "seq_lens");
  g.batch = small(lens.numel(), "requests");
  g.num_queries = small(way.numel(), "nodes");
  g.num_q_heads = g.num_kv_heads;
  g.softmax_scale = 1.f;
  const int32_t *path = c.ints(way, g.num_queries, "path"), *seq_lens = c.ints(lens, g.batch, "seq_lens"), *q_start = c.ints_or_none(a[2], (int64_t)g.batch + 1, "q_start"),
                *table = c.table(a[3], g.batch, g.max_pages_per_seq, g.page_table_stride);
  void* const stream = c.stream(a[8]);
  return without_gil([&] { return g_keep(&g, layers, path, seq_lens, q_start, table, cache.k, cache.v, cache.k_scales, cache.v_scales, stream); });
}

// The library's code, or a Python error.
template <int (*F)(PyObject* const*), int ARGS>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != ARGS) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    const int rc = F(a);
    return PyLong_FromLong(rc);
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "a tensor could not be read");
  }
  return nullptr;
}

// OmniAttnError, current device, current stream of a device, addresses of the library's functions
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 12) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  PyObject** const keep[3] = {&g_error, &g_device, &g_stream};
  for (int i = 0; i < 3; ++i) {
    Py_INCREF(a[i]);
    Py_XDECREF(*keep[i]);
    *keep[i] = a[i];
  }
  g_extend = reinterpret_cast<decltype(g_extend)>(PyLong_AsVoidPtr(a[3]));
  g_release = reinterpret_cast<decltype(g_release)>(PyLong_AsVoidPtr(a[4]));
  g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[5]));
  g_decode = reinterpret_cast<decltype(g_decode)>(PyLong_AsVoidPtr(a[6]));
  g_truncate = reinterpret_cast<decltype(g_truncate)>(PyLong_AsVoidPtr(a[7]));
  g_tree_masks = reinterpret_cast<decltype(g_tree_masks)>(PyLong_AsVoidPtr(a[8]));
  g_tree = reinterpret_cast<decltype(g_tree)>(PyLong_AsVoidPtr(a[9]));
  g_verify = reinterpret_cast<decltype(g_verify)>(PyLong_AsVoidPtr(a[10]));
  g_keep = reinterpret_cast<decltype(g_keep)>(PyLong_AsVoidPtr(a[11]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

#define OA_ENTRY(name, args) {#name, (PyCFunction)(void*)(entry<name, args>), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {OA_ENTRY(extend, 10), OA_ENTRY(release, 6), OA_ENTRY(append, 8), OA_ENTRY(decode, 15), OA_ENTRY(truncate, 8),
                           OA_ENTRY(tree_masks, 6), OA_ENTRY(tree, 16), OA_ENTRY(verify, 13), OA_ENTRY(keep, 9),
                           {"setup", (PyCFunction)(void*)setup, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "gqa_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_gqa_marshal(void) {
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  return s_cuda_stream ? PyModule_Create(&g_module) : nullptr;
}
