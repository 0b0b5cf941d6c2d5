// Argument marshalling of the per-layer operators (per-head norm with rotation, 4-bit paged cache, 4-bit weights) and of
// those that choose tokens, for torch tensors:
// checks types, shapes and strides, allocates what the caller did not pass, and calls the C entry points of
// include/thinfer.h on the tensors' device and its current stream.  No arithmetic happens here.
//
// These operators run once per layer and decode step on small tensors, where the checks of eight tensors, two
// allocations and twenty foreign-function arguments cost more in the interpreter (10 to 17 us) than the kernels take.
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/thinfer.h"

namespace {

PyObject* g_error = nullptr;   // ThinferError(code, text)

struct Api {
  decltype(&thinfer_op_qk_norm_rope) qk_norm_rope = nullptr;
  decltype(&thinfer_op_kv4_reserve) reserve = nullptr;
  decltype(&thinfer_op_kv4_append) append = nullptr;
  decltype(&thinfer_op_kv4_read) read = nullptr;
  decltype(&thinfer_kv4_attention_workspace) attention_workspace = nullptr;
  decltype(&thinfer_op_kv4_attention) attention = nullptr;
  decltype(&thinfer_kv4_pages_workspace) pages_workspace = nullptr;
  decltype(&thinfer_op_kv4_fork) fork = nullptr;
  decltype(&thinfer_op_kv4_compact) compact = nullptr;
  decltype(&thinfer_w4_bytes) w4_bytes = nullptr;
  decltype(&thinfer_op_w4_quantize) w4_quantize = nullptr;
  decltype(&thinfer_op_w4_read) w4_read = nullptr;
  decltype(&thinfer_w4_linear_workspace) w4_linear_workspace = nullptr;
  decltype(&thinfer_op_w4_linear) w4_linear = nullptr;
  decltype(&thinfer_op_token_probs) token_probs = nullptr;
  decltype(&thinfer_op_verify_drafts) verify_drafts = nullptr;
  decltype(&thinfer_last_error) last_error = nullptr;
};
Api g_api[2];   // FP16 build, BF16 build

struct Refusal {
  int code;
  std::string text;
};
[[noreturn]] void refuse(const std::string& text) { throw Refusal{THINFER_EINVAL, text}; }
void check(const Api& api, int rc) {
  if (rc != THINFER_OK) {
    const char* text = api.last_error(nullptr);
    throw Refusal{rc, text ? text : ""};
  }
}

// Makes one call of the library without the interpreter lock: a full launch queue makes it wait, and the process's other
// threads go on meanwhile, as they do around a foreign function.  The arguments are ready before the lock is given up.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F, typename... A>
void call(const Api& api, F f, A... a) {
  int rc;
  {
    const Unlocked now;
    rc = f(a...);
  }
  check(api, rc);
}

std::string describe(const at::Tensor& t) {
  std::string s = std::string(c10::toString(t.scalar_type())) + " [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + "] on " + t.device().str();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is wanted");
  return THPVariable_Unpack(o);
}
int64_t number(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse(std::string(name) + ": a whole number is wanted");
  }
  return v;
}
bool truth(PyObject* o, const char* name) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) {
    PyErr_Clear();
    refuse(std::string(name) + ": a truth value is wanted");
  }
  return v == 1;
}
int32_t small(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(name) + " = " + std::to_string(v) + " does not fit 32 bits");
  return static_cast<int32_t>(v);
}

// The device of a call: checked, made current, its current stream.
struct On {
  c10::Device device;
  c10::cuda::OptionalCUDAGuard guard;
  void* stream = nullptr;
  explicit On(const at::Tensor& t) : device(t.device()) {
    if (!t.is_cuda()) refuse("tensors must be on a CUDA device, not " + device.str());
    if (c10::cuda::current_device() != device.index()) guard.set_device(device);
    stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
  }
  // A new contiguous tensor of this device, straight from its allocator.
  at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const { return at::detail::empty_cuda(shape, type, device, c10::nullopt); }
  // Memory for the length of a call: given back to the stream's pool when it returns, as a tensor's would be.
  c10::DataPtr scratch(size_t bytes) const { return c10::cuda::CUDACachingAllocator::get()->allocate(bytes); }
};

const Api& api_of(at::ScalarType t) {
  if (t == at::kHalf) return g_api[0];
  if (t == at::kBFloat16) return g_api[1];
  throw Refusal{THINFER_EUNSUPPORTED, std::string("storage type ") + c10::toString(t) + ": the library is built for float16 and bfloat16"};
}

void* plain(const at::Tensor& t, const char* name, const On& on, at::IntArrayRef shape, at::ScalarType type = at::kInt) {
  if (t.scalar_type() != type || t.device() != on.device || !t.sizes().equals(shape) || !t.is_contiguous()) {
    std::string want = std::string(name) + ": a contiguous " + c10::toString(type) + " tensor [";
    for (size_t i = 0; i < shape.size(); ++i) want += (i ? ", " : "") + std::to_string(shape[i]);
    refuse(want + "] on " + on.device.str() + ", not " + describe(t));
  }
  return t.data_ptr();
}

// Elements between the tokens of [tokens, heads, head_dim] whose heads lie side by side.
int64_t token_stride(const at::Tensor& t, const char* name, at::ScalarType type, const On& on) {
  if (t.dim() != 3 || t.scalar_type() != type || t.device() != on.device)
    refuse(std::string(name) + ": a " + c10::toString(type) + " tensor [tokens, heads, head_dim] on " + on.device.str() + ", not " + describe(t));
  const int64_t n = t.size(0), h = t.size(1), d = t.size(2);
  if (n == 0 || h == 0 || t.stride(2) != 1 || (h != 1 && t.stride(1) != d))
    refuse(std::string(name) + ": the heads of a token must be contiguous, and there must be some");
  return n > 1 ? t.stride(0) : h * d;
}

void same_shape(const at::Tensor& a, const at::Tensor& b, const char* what) {
  if (!a.sizes().equals(b.sizes())) refuse(what);
}

// Number of KV heads of a uint8 pool whose last dimension is a page.
int64_t pool_heads(const at::Tensor& pool, int64_t dims, int64_t page, int64_t d, const On& on) {
  if (pool.scalar_type() != at::kByte || pool.dim() != dims || pool.device() != on.device || !pool.is_contiguous())
    refuse("pool: a contiguous uint8 tensor of " + std::to_string(dims) + " dimensions on " + on.device.str() + ", not " + describe(pool));
  if (page <= 0 || page > 1 << 20 || d <= 0 || d > 1 << 20) refuse("page_size and head_dim must be positive");
  const int64_t per = page * (d + 8), bytes = pool.size(dims - 1), heads = bytes / per;
  if (heads == 0 || heads * per != bytes) refuse("pool: a page has a multiple of " + std::to_string(per) + " bytes, not " + std::to_string(bytes));
  return heads;
}

const int32_t* table_of(const at::Tensor& t, const On& on) {
  if (t.dim() != 2) refuse("table: int32 [rows, max_pages]");
  return static_cast<const int32_t*>(plain(t, "table", on, t.sizes()));
}

template <typename F>
at::Tensor given_or(PyObject* o, const char* name, F make) {
  return o == Py_None ? make() : tensor(o, name);
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* pack(std::initializer_list<at::Tensor> ts) {
  PyObject* out = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) PyTuple_SET_ITEM(out, i++, wrap(t));
  return out;
}

// q, k, q_gain, k_gain, eps, turns, positions, halves, q_out, k_out
PyObject* qk_norm_rope(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &gq = tensor(a[2], "q_gain"), &gk = tensor(a[3], "k_gain");
  const at::Tensor &turns = tensor(a[5], "turns"), &positions = tensor(a[6], "positions");
  const On on(q);
  const double eps = PyFloat_AsDouble(a[4]);
  if (eps == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse("eps: a number is wanted");
  }
  const at::ScalarType type = q.scalar_type();
  const Api& api = api_of(type);
  const int64_t qs = token_stride(q, "q", type, on), ks = token_stride(k, "k", type, on);
  const int64_t n = q.size(0), hq = q.size(1), d = q.size(2), hkv = k.size(1);
  if (k.size(0) != n || k.size(2) != d) refuse("q and k must agree in tokens and head_dim");
  if (turns.dim() != 1) refuse("turns: FP64 [rotary_dim / 2]");
  const at::Tensor q_out = given_or(a[8], "q_out", [&] { return on.empty({n, hq, d}, type); });
  const at::Tensor k_out = given_or(a[9], "k_out", [&] { return on.empty({n, hkv, d}, type); });
  same_shape(q_out, q, "q_out: the shape of q");
  same_shape(k_out, k, "k_out: the shape of k");
  const int64_t qos = token_stride(q_out, "q_out", type, on), kos = token_stride(k_out, "k_out", type, on);
  call(api, api.qk_norm_rope, q.data_ptr(), qs, k.data_ptr(), ks, q_out.data_ptr(), qos, k_out.data_ptr(), kos, plain(gq, "q_gain", on, {d}, type),
                              plain(gk, "k_gain", on, {d}, type), static_cast<const double*>(plain(turns, "turns", on, turns.sizes(), at::kDouble)),
                              static_cast<const int32_t*>(plain(positions, "positions", on, {n})), small(n, "tokens"), small(hq, "heads"),
                              small(hkv, "heads"), small(d, "head_dim"), small(2 * turns.size(0), "rotary_dim"), truth(a[7], "halves"),
                              static_cast<float>(eps), on.stream);
  return pack({q_out, k_out});
}

// table, lens, add, n_pages, page_size, lens_out, refused
PyObject* reserve(PyObject* const* a) {
  const at::Tensor &table = tensor(a[0], "table"), &lens = tensor(a[1], "lens"), &add = tensor(a[2], "add");
  const On on(table);
  const int32_t* tab = table_of(table, on);
  const int64_t rows = table.size(0);
  const at::Tensor lens_out = given_or(a[5], "lens_out", [&] { return on.empty({rows}, at::kInt); });
  const at::Tensor refused = given_or(a[6], "refused", [&] { return on.empty({1}, at::kLong); });
  call(g_api[0], g_api[0].reserve, const_cast<int32_t*>(tab), static_cast<const int32_t*>(plain(lens, "lens", on, {rows})),
                                   static_cast<const int32_t*>(plain(add, "add", on, {rows})),
                                   static_cast<int32_t*>(plain(lens_out, "lens_out", on, {rows})),
                                   static_cast<int64_t*>(plain(refused, "refused", on, {1}, at::kLong)), small(rows, "rows"),
                                   small(table.size(1), "max_pages"), small(number(a[3], "n_pages"), "n_pages"),
                                   small(number(a[4], "page_size"), "page_size"), on.stream);
  return pack({lens_out, refused});
}

// pool, table, k, v, rows, positions, page_size
PyObject* append(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0], "pool"), &table = tensor(a[1], "table"), &k = tensor(a[2], "k"), &v = tensor(a[3], "v");
  const at::Tensor &rows = tensor(a[4], "rows"), &positions = tensor(a[5], "positions");
  const On on(pool);
  const int64_t page = number(a[6], "page_size");
  const at::ScalarType type = k.scalar_type();
  const Api& api = api_of(type);
  const int64_t ks = token_stride(k, "k", type, on), vs = token_stride(v, "v", type, on);
  same_shape(k, v, "k and v must have one shape");
  const int64_t n = k.size(0), hkv = k.size(1), d = k.size(2);
  if (pool_heads(pool, 2, page, d, on) != hkv) refuse("the pool's pages are for another number of heads");
  call(api, api.append, pool.data_ptr(), small(pool.size(0), "pages"), table_of(table, on), small(table.size(0), "rows"), small(table.size(1), "max_pages"),
                        k.data_ptr(), ks, v.data_ptr(), vs, static_cast<const int32_t*>(plain(rows, "rows", on, {n})),
                        static_cast<const int32_t*>(plain(positions, "positions", on, {n})), small(n, "tokens"), small(hkv, "heads"),
                        small(d, "head_dim"), small(page, "page_size"), on.stream);
  Py_RETURN_NONE;
}

// pool, table, rows, positions, page_size, head_dim, bf16 (truth value), k_out, v_out
PyObject* read(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0], "pool"), &table = tensor(a[1], "table"), &rows = tensor(a[2], "rows"), &positions = tensor(a[3], "positions");
  const On on(pool);
  const int64_t page = number(a[4], "page_size"), d = number(a[5], "head_dim"), hkv = pool_heads(pool, 2, page, d, on), n = positions.numel();
  const at::ScalarType type = truth(a[6], "bf16") ? at::kBFloat16 : at::kHalf;
  const Api& api = api_of(type);
  const at::Tensor k_out = given_or(a[7], "k_out", [&] { return on.empty({n, hkv, d}, type); });
  const at::Tensor v_out = given_or(a[8], "v_out", [&] { return at::empty_strided({n, hkv, d}, k_out.strides(), k_out.options()); });
  const int64_t shape[3] = {n, hkv, d};
  for (const at::Tensor* t : {&k_out, &v_out})
    if (!t->sizes().equals(shape) || t->scalar_type() != type || t->device() != on.device || (d > 1 && t->stride(2) != 1) ||
        (n > 1 && t->stride(0) != k_out.stride(0)) || (hkv > 1 && t->stride(1) != k_out.stride(1)))
      refuse("k_out, v_out: [tokens, heads, head_dim] of one type, device and strides, the values of a head contiguous");
  // the stride of a dimension of one says nothing
  const int64_t hs = hkv > 1 ? k_out.stride(1) : d, ts = n > 1 ? k_out.stride(0) : hkv * d;
  call(api, api.read, pool.data_ptr(), small(pool.size(0), "pages"), table_of(table, on), small(table.size(0), "rows"), small(table.size(1), "max_pages"),
                      k_out.data_ptr(), v_out.data_ptr(), ts, hs, static_cast<const int32_t*>(plain(rows, "rows", on, {n})),
                      static_cast<const int32_t*>(plain(positions, "positions", on, {n})), small(n, "tokens"), small(hkv, "heads"),
                      small(d, "head_dim"), small(page, "page_size"), on.stream);
  return pack({k_out, v_out});
}

// q, pool, table, lens, page_size, out, workspace
PyObject* attention(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0], "q"), &pool = tensor(a[1], "pool"), &table = tensor(a[2], "table"), &lens = tensor(a[3], "lens");
  const On on(q);
  const int64_t page = number(a[4], "page_size");
  const at::ScalarType type = q.scalar_type();
  const Api& api = api_of(type);
  if (q.dim() != 4) refuse("q: [batch, queries, n_q_heads, head_dim]");
  const int64_t b = q.size(0), n = q.size(1), hq = q.size(2), d = q.size(3);
  if (b * n * hq == 0 || q.stride(3) != 1 || (hq != 1 && q.stride(2) != d) || (n > 1 && b > 1 && q.stride(0) != n * q.stride(1)))
    refuse("q: the heads of a token must be contiguous and the query tokens evenly spaced");
  const int64_t qs = n > 1 ? q.stride(1) : b > 1 ? q.stride(0) : hq * d;
  const int64_t hkv = pool_heads(pool, 2, page, d, on);
  const int32_t* tab = table_of(table, on);
  if (table.size(0) != b) refuse("table: one row per request");
  const at::Tensor out = given_or(a[5], "out", [&] { return on.empty({b, n, hq, d}, type); });
  c10::DataPtr own;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (a[6] == Py_None) {
    check(api, api.attention_workspace(small(b, "batch"), small(n, "queries"), small(hq, "heads"), small(hkv, "heads"), small(d, "head_dim"), &ws_bytes));
    own = on.scratch(ws_bytes);
    ws = own.get();
  } else {
    const at::Tensor& given = tensor(a[6], "workspace");
    ws_bytes = static_cast<size_t>(given.numel());
    ws = plain(given, "workspace", on, {given.numel()}, at::kByte);
  }
  call(api, api.attention, q.data_ptr(), qs, pool.data_ptr(), small(pool.size(0), "pages"), tab, small(table.size(1), "max_pages"),
                           static_cast<const int32_t*>(plain(lens, "lens", on, {b})), plain(out, "out", on, {b, n, hq, d}, type), small(b, "batch"),
                           small(n, "queries"), small(hq, "heads"), small(hkv, "heads"), small(d, "head_dim"), small(page, "page_size"),
                           ws, ws_bytes, on.stream);
  return wrap(out);
}

c10::DataPtr pages_workspace(int64_t rows, int64_t n_pages, const On& on, size_t* bytes) {
  check(g_api[0], g_api[0].pages_workspace(small(rows, "rows"), small(n_pages, "pages"), bytes));
  return on.scratch(*bytes);
}

// pool, table, lens, source, page_size, head_dim, table_out, lens_out, refused
PyObject* fork(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0], "pool"), &table = tensor(a[1], "table"), &lens = tensor(a[2], "lens"), &source = tensor(a[3], "source");
  const On on(pool);
  const int64_t page = number(a[4], "page_size"), d = number(a[5], "head_dim"), hkv = pool_heads(pool, 3, page, d, on);
  const int32_t* tab = table_of(table, on);
  const int64_t rows = table.size(0), width = table.size(1);
  const at::Tensor table_out = given_or(a[6], "table_out", [&] { return on.empty({rows, width}, at::kInt); });
  const at::Tensor lens_out = given_or(a[7], "lens_out", [&] { return on.empty({rows}, at::kInt); });
  const at::Tensor refused = given_or(a[8], "refused", [&] { return on.empty({1}, at::kLong); });
  size_t ws_bytes = 0;
  const c10::DataPtr ws = pages_workspace(rows, pool.size(1), on, &ws_bytes);
  call(g_api[0], g_api[0].fork, pool.data_ptr(), small(pool.size(0), "layers"), small(pool.size(1), "pages"), tab,
                                static_cast<const int32_t*>(plain(lens, "lens", on, {rows})), static_cast<const int32_t*>(plain(source, "source", on, {rows})),
                                static_cast<int32_t*>(plain(table_out, "table_out", on, {rows, width})),
                                static_cast<int32_t*>(plain(lens_out, "lens_out", on, {rows})),
                                static_cast<int64_t*>(plain(refused, "refused", on, {1}, at::kLong)), small(rows, "rows"), small(width, "max_pages"),
                                small(hkv, "heads"), small(d, "head_dim"), small(page, "page_size"), ws.get(), ws_bytes, on.stream);
  return pack({table_out, lens_out, refused});
}

// pool, table, lens, page_size, head_dim, table_out, live
PyObject* compact(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0], "pool"), &table = tensor(a[1], "table"), &lens = tensor(a[2], "lens");
  const On on(pool);
  const int64_t page = number(a[3], "page_size"), d = number(a[4], "head_dim"), hkv = pool_heads(pool, 3, page, d, on);
  const int32_t* tab = table_of(table, on);
  const int64_t rows = table.size(0), width = table.size(1);
  const at::Tensor table_out = given_or(a[5], "table_out", [&] { return on.empty({rows, width}, at::kInt); });
  const at::Tensor live = given_or(a[6], "live", [&] { return on.empty({1}, at::kLong); });
  size_t ws_bytes = 0;
  const c10::DataPtr ws = pages_workspace(rows, pool.size(1), on, &ws_bytes);
  call(g_api[0], g_api[0].compact, pool.data_ptr(), small(pool.size(0), "layers"), small(pool.size(1), "pages"), tab,
                                   static_cast<const int32_t*>(plain(lens, "lens", on, {rows})),
                                   static_cast<int32_t*>(plain(table_out, "table_out", on, {rows, width})),
                                   static_cast<int64_t*>(plain(live, "live", on, {1}, at::kLong)), small(rows, "rows"), small(width, "max_pages"),
                                   small(hkv, "heads"), small(d, "head_dim"), small(page, "page_size"), ws.get(), ws_bytes,
                                   on.stream);
  return pack({table_out, live});
}

// Elements between the rows of [rows, columns] whose columns lie side by side; a stride of a single row says nothing.
int64_t row_stride(const at::Tensor& t, const char* name, at::ScalarType type, const On& on) {
  if (t.dim() != 2 || t.scalar_type() != type || t.device() != on.device)
    refuse(std::string(name) + ": a " + c10::toString(type) + " tensor [rows, columns] on " + on.device.str() + ", not " + describe(t));
  if (t.size(0) == 0 || t.size(1) == 0 || (t.size(1) != 1 && t.stride(1) != 1))
    refuse(std::string(name) + ": the columns of a row must be contiguous, and there must be some");
  return t.size(0) > 1 ? t.stride(0) : t.size(1);
}

void* packed_weights(const at::Tensor& t, const Api& api, int64_t n, int64_t k, int64_t group, const On& on) {
  size_t bytes = 0;
  check(api, api.w4_bytes(small(n, "n_out"), small(k, "k"), small(group, "group"), &bytes));
  return plain(t, "packed", on, {static_cast<int64_t>(bytes)}, at::kByte);
}

// w, group, packed
PyObject* w4_quantize(PyObject* const* a) {
  const at::Tensor& w = tensor(a[0], "w");
  const On on(w);
  const Api& api = api_of(w.scalar_type());
  const int64_t ws = row_stride(w, "w", w.scalar_type(), on), n = w.size(0), k = w.size(1), group = number(a[1], "group");
  size_t bytes = 0;
  check(api, api.w4_bytes(small(n, "n_out"), small(k, "k"), small(group, "group"), &bytes));
  const at::Tensor packed = given_or(a[2], "packed", [&] { return on.empty({static_cast<int64_t>(bytes)}, at::kByte); });
  call(api, api.w4_quantize, w.data_ptr(), ws, packed_weights(packed, api, n, k, group, on), small(n, "n_out"), small(k, "k"), small(group, "group"), on.stream);
  return wrap(packed);
}

// packed, n_out, k, group, bf16 (truth value), out
PyObject* w4_read(PyObject* const* a) {
  const at::Tensor& packed = tensor(a[0], "packed");
  const On on(packed);
  const int64_t n = number(a[1], "n_out"), k = number(a[2], "k"), group = number(a[3], "group");
  const at::ScalarType type = truth(a[4], "bf16") ? at::kBFloat16 : at::kHalf;
  const Api& api = api_of(type);
  const void* in = packed_weights(packed, api, n, k, group, on);
  const at::Tensor out = given_or(a[5], "out", [&] { return on.empty({n, k}, type); });
  const int64_t os = row_stride(out, "out", type, on);
  if (out.size(0) != n || out.size(1) != k) refuse("out: [n_out, k]");
  call(api, api.w4_read, in, out.data_ptr(), os, small(n, "n_out"), small(k, "k"), small(group, "group"), on.stream);
  return wrap(out);
}

// x, packed, n_out, group, out_fp32, out, workspace
PyObject* w4_linear(PyObject* const* a) {
  const at::Tensor &x = tensor(a[0], "x"), &packed = tensor(a[1], "packed");
  const On on(x);
  const at::ScalarType type = x.scalar_type();
  const Api& api = api_of(type);
  const int64_t xs = row_stride(x, "x", type, on), rows = x.size(0), k = x.size(1), n = number(a[2], "n_out"), group = number(a[3], "group");
  const void* weights = packed_weights(packed, api, n, k, group, on);
  bool fp32 = truth(a[4], "out_fp32");
  const at::Tensor out = given_or(a[5], "out", [&] { return on.empty({rows, n}, fp32 ? at::kFloat : type); });
  if (a[5] != Py_None) fp32 = out.scalar_type() == at::kFloat;
  const int64_t os = row_stride(out, "out", fp32 ? at::kFloat : type, on);
  if (out.size(0) != rows || out.size(1) != n) refuse("out: [rows, n_out]");
  c10::DataPtr own;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (a[6] == Py_None) {
    check(api, api.w4_linear_workspace(small(rows, "rows"), small(n, "n_out"), small(k, "k"), small(group, "group"), &ws_bytes));
    if (ws_bytes > 0) own = on.scratch(ws_bytes);
    ws = own.get();
  } else {
    const at::Tensor& given = tensor(a[6], "workspace");
    ws_bytes = static_cast<size_t>(given.numel());
    ws = plain(given, "workspace", on, {given.numel()}, at::kByte);
  }
  call(api, api.w4_linear, x.data_ptr(), xs, weights, out.data_ptr(), os, small(rows, "rows"), small(n, "n_out"), small(k, "k"), small(group, "group"),
                           fp32 ? 1 : 0, ws, ws_bytes, on.stream);
  return wrap(out);
}

// logits, temperature, out
PyObject* token_probs(PyObject* const* a) {
  const at::Tensor& logits = tensor(a[0], "logits");
  const On on(logits);
  const int64_t ls = row_stride(logits, "logits", at::kFloat, on), rows = logits.size(0), vocab = logits.size(1);
  const float* temperature = a[1] == Py_None ? nullptr : static_cast<const float*>(plain(tensor(a[1], "temperature"), "temperature", on, {rows}, at::kFloat));
  const at::Tensor out = given_or(a[2], "out", [&] { return on.empty({rows, vocab}, at::kFloat); });
  same_shape(out, logits, "out: the shape of the logits");
  const int64_t os = row_stride(out, "out", at::kFloat, on);
  call(g_api[0], g_api[0].token_probs, static_cast<const float*>(logits.data_ptr()), ls, temperature, static_cast<float*>(out.data_ptr()), os, small(rows, "rows"),
                                       small(vocab, "vocab"), on.stream);
  return wrap(out);
}

// [batch, rows, vocab] whose values of a row lie side by side
const float* distributions(const at::Tensor& t, const char* name, int64_t batch, int64_t rows, int64_t vocab, const On& on) {
  if (t.dim() != 3 || t.scalar_type() != at::kFloat || t.device() != on.device || t.size(0) != batch || t.size(1) != rows || t.size(2) != vocab ||
      (vocab > 1 && t.stride(2) != 1))
    refuse(std::string(name) + ": a Float tensor [" + std::to_string(batch) + ", " + std::to_string(rows) + ", " + std::to_string(vocab) +
           "] with contiguous rows on " + on.device.str() + ", not " + describe(t));
  return static_cast<const float*>(t.data_ptr());
}

// p, q, drafts, uniforms, counts, tokens, accepted
PyObject* verify_drafts(PyObject* const* a) {
  const at::Tensor &p = tensor(a[0], "p"), &drafts = tensor(a[2], "drafts"), &uniforms = tensor(a[3], "uniforms");
  const On on(p);
  if (p.dim() != 3 || p.numel() == 0) refuse("p: [batch, drafts + 1, vocab], with something in it");
  const int64_t b = p.size(0), n = p.size(1) - 1, v = p.size(2);
  const float *pp = distributions(p, "p", b, n + 1, v, on), *qp = nullptr;
  int64_t qb = 0, qr = 0;
  if (a[1] != Py_None && n > 0) {
    const at::Tensor& q = tensor(a[1], "q");
    qp = distributions(q, "q", b, n, v, on);
    qb = b > 1 ? q.stride(0) : 0;
    qr = n > 1 ? q.stride(1) : 0;
  }
  const int32_t* counts = a[4] == Py_None ? nullptr : static_cast<const int32_t*>(plain(tensor(a[4], "counts"), "counts", on, {b}));
  const at::Tensor tokens = given_or(a[5], "tokens", [&] { return on.empty({b, n + 1}, at::kInt); });
  const at::Tensor accepted = given_or(a[6], "accepted", [&] { return on.empty({b}, at::kInt); });
  call(g_api[0], g_api[0].verify_drafts, pp, b > 1 ? p.stride(0) : 0, n > 0 ? p.stride(1) : 0, qp, qb, qr,
                                         static_cast<const int32_t*>(plain(drafts, "drafts", on, {b, n})),
                                         static_cast<const float*>(plain(uniforms, "uniforms", on, {b, n + 1}, at::kFloat)), counts,
                                         static_cast<int32_t*>(plain(tokens, "tokens", on, {b, n + 1})),
                                         static_cast<int32_t*>(plain(accepted, "accepted", on, {b})), small(b, "batch"), small(n, "drafts"),
                                         small(v, "vocab"), on.stream);
  return pack({tokens, accepted});
}

// No C++ exception passes this frame: a refusal becomes ThinferError(code, text), what torch throws becomes torch's error.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N || g_error == nullptr) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd, after bind()", N, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Refusal& r) {
    PyObject* e = PyObject_CallFunction(g_error, "is", r.code, r.text.c_str());
    if (e != nullptr) {
      PyErr_SetObject(g_error, e);
      Py_DECREF(e);
    }
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// bind(error class, addresses of the FP16 build, of the BF16 build): the entry points in the order of Api
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *error, *tables[2];
  if (!PyArg_ParseTuple(args, "OOO", &error, &tables[0], &tables[1])) return nullptr;
  for (int s = 0; s < 2; ++s) {
    constexpr int kCount = 17;
    void* at[kCount];
    if (PySequence_Size(tables[s]) != kCount) {
      PyErr_Format(PyExc_TypeError, "%d addresses", kCount);
      return nullptr;
    }
    for (int i = 0; i < kCount; ++i) {
      PyObject* o = PySequence_GetItem(tables[s], i);
      at[i] = o ? PyLong_AsVoidPtr(o) : nullptr;
      Py_XDECREF(o);
      if (at[i] == nullptr) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is NULL");
        return nullptr;
      }
    }
    Api& p = g_api[s];
    p.qk_norm_rope = reinterpret_cast<decltype(p.qk_norm_rope)>(at[0]);
    p.reserve = reinterpret_cast<decltype(p.reserve)>(at[1]);
    p.append = reinterpret_cast<decltype(p.append)>(at[2]);
    p.read = reinterpret_cast<decltype(p.read)>(at[3]);
    p.attention_workspace = reinterpret_cast<decltype(p.attention_workspace)>(at[4]);
    p.attention = reinterpret_cast<decltype(p.attention)>(at[5]);
    p.pages_workspace = reinterpret_cast<decltype(p.pages_workspace)>(at[6]);
    p.fork = reinterpret_cast<decltype(p.fork)>(at[7]);
    p.compact = reinterpret_cast<decltype(p.compact)>(at[8]);
    p.w4_bytes = reinterpret_cast<decltype(p.w4_bytes)>(at[9]);
    p.w4_quantize = reinterpret_cast<decltype(p.w4_quantize)>(at[10]);
    p.w4_read = reinterpret_cast<decltype(p.w4_read)>(at[11]);
    p.w4_linear_workspace = reinterpret_cast<decltype(p.w4_linear_workspace)>(at[12]);
    p.w4_linear = reinterpret_cast<decltype(p.w4_linear)>(at[13]);
    p.token_probs = reinterpret_cast<decltype(p.token_probs)>(at[14]);
    p.verify_drafts = reinterpret_cast<decltype(p.verify_drafts)>(at[15]);
    p.last_error = reinterpret_cast<decltype(p.last_error)>(at[16]);
  }
  Py_INCREF(error);
  Py_XDECREF(g_error);
  g_error = error;
  Py_RETURN_NONE;
}

#define ENTRY(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {ENTRY(qk_norm_rope, 10), ENTRY(reserve, 7), ENTRY(append, 7), ENTRY(read, 9), ENTRY(attention, 7),
                          ENTRY(fork, 9), ENTRY(compact, 7), ENTRY(w4_quantize, 3), ENTRY(w4_read, 6), ENTRY(w4_linear, 7),
                          ENTRY(token_probs, 3), ENTRY(verify_drafts, 7), {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops(void) { return PyModule_Create(&kModule); }
