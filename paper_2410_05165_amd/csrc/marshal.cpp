// The calls of paged.py on PyTorch tensors: checks of types, shapes, devices and strides,
// new outputs, and the arguments of the C entry points, nothing else.  These calls come
// once a layer and the small ones take 4 to 5 us on the GPU.  A call takes on the host,
// launch included (3.6 us), with the checks in Python and here: page plan 14.3 and 6.9 us,
// append 7.4 and 3.7, tree attention 13.8 and 5.9, logit rules 13.8 and 5.0.
//
// Every function takes positional arguments, the raw stream last, and raises ValueError
// for a tensor that does not fit and AtspeedError for a status.
#include <Python.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <limits>
#include <string>
#include <utility>

#include <ATen/core/Tensor.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/atspeed.h"

namespace {

PyObject* g_error = nullptr;   // AtspeedError

struct Raised {};                           // a Python error is set
[[noreturn]] void bad(const std::string& msg) {
  PyErr_SetString(PyExc_ValueError, msg.c_str());
  throw Raised{};
}

void check(atspeed_status s) {
  if (s == ATSPEED_OK) return;
  PyObject* args = Py_BuildValue("(is)", (int)s, atspeed_last_error());
  if (args) {
    PyErr_SetObject(g_error, args);
    Py_DECREF(args);
  }
  throw Raised{};
}

// A launch waits where the stream's queue is full: other threads run meanwhile.
template <class F>
void enqueue(F&& call) {
  PyThreadState* state = PyEval_SaveThread();
  const atspeed_status s = call();
  PyEval_RestoreThread(state);
  check(s);
}

std::string shown(c10::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) bad(std::string(name) + ": want a tensor");
  return THPVariable_Unpack(o);
}

const at::Tensor& gpu_tensor(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) bad(std::string(name) + " is on " + t.device().str() + ": the operators run on the GPU alone");
  return t;
}

template <class T>
T* address(const at::Tensor& t) {
  return static_cast<T*>(const_cast<void*>(t.unsafeGetTensorImpl()->data()));
}

// A call writes to this tensor (None: none): autograd, which sees nothing of it, refuses a
// backward pass that saved it before.
void written(PyObject* o) {
  if (o == Py_None) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The address of a contiguous tensor of this type and shape on this GPU (None: null).
template <class T>
T* want(PyObject* o, const char* name, c10::ScalarType type, std::initializer_list<int64_t> shape, const at::Device& dev) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() == type && t.sizes() == c10::IntArrayRef(shape) && t.device() == dev && t.is_contiguous())
    return address<T>(t);
  bad(std::string(name) + ": want a contiguous " + c10::toString(type) + " " + shown(shape) + " on " + dev.str() + ", got " +
      c10::toString(t.scalar_type()) + " " + shown(t.sizes()) + " on " + t.device().str());
}
int32_t* want_i32(PyObject* o, const char* name, std::initializer_list<int64_t> shape, const at::Device& dev) {
  return want<int32_t>(o, name, c10::ScalarType::Int, shape, dev);
}

int32_t int32(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v < std::numeric_limits<int32_t>::min() || v > std::numeric_limits<int32_t>::max())
    bad(std::string(name) + " is out of range");
  return (int32_t)v;
}
int32_t int32(int64_t v, const char* name) {
  if (v > std::numeric_limits<int32_t>::max()) bad(std::string(name) + " is too large");
  return (int32_t)v;
}
void* stream_of(PyObject* o) {
  void* s = PyLong_AsVoidPtr(o);
  if (!s && PyErr_Occurred()) throw Raised{};
  return s;
}
bool flag(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}
float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return (float)v;
}

int32_t dtype_of(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == c10::ScalarType::Float) return ATSPEED_FP32;
  if (t.scalar_type() == c10::ScalarType::BFloat16) return ATSPEED_BF16;
  bad(std::string(name) + ": want float32 or bfloat16");
}

// The stride of a dimension of one element says nothing.
int64_t stride(const at::Tensor& t, int64_t i) { return t.size(i) > 1 ? t.stride(i) : 0; }

struct Caches {
  at::Device dev;
  c10::ScalarType type;
  int32_t dtype, pool, page, heads, dh;
  atspeed_pages k, v;
};
Caches caches(PyObject* ko, PyObject* vo) {
  const at::Tensor& k = gpu_tensor(ko, "k_cache");
  const at::Tensor& v = tensor(vo, "v_cache");
  if (k.dim() != 4) bad("k_cache: want [pages, page_size, kv_heads, d_head]");
  if (v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type() || v.device() != k.device() || k.stride(3) != 1 ||
      v.stride(3) != 1)
    bad("the caches want one type, shape and device, the last dimension contiguous");
  Caches c{k.device(), k.scalar_type(), dtype_of(k, "k_cache"), int32(k.size(0), "pages"), int32(k.size(1), "page_size"),
           int32(k.size(2), "kv_heads"), int32(k.size(3), "d_head"),
           {address<void>(k), stride(k, 0), stride(k, 1), stride(k, 2)},
           {address<void>(v), stride(v, 0), stride(v, 1), stride(v, 2)}};
  return c;
}

// Rows [n, heads, d_head] with any row and head strides.
const at::Tensor& rows_of(PyObject* o, const char* name, int64_t n, int64_t heads, const Caches& c) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != c.dh || t.scalar_type() != c.type ||
      t.device() != c.dev || t.stride(2) != 1)
    bad(std::string(name) + ": want " + c10::toString(c.type) + " " + shown({n, heads, c.dh}) + " on " + c.dev.str() +
        ", the last dimension contiguous, got " + c10::toString(t.scalar_type()) + " " + shown(t.sizes()) + " on " +
        t.device().str());
  return t;
}

template <class F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t wanted, F&& f) {
  if (got != wanted) {
    PyErr_Format(PyExc_TypeError, "want %zd arguments, got %zd", wanted, got);
    return nullptr;
  }
  try {
    at::AutoDispatchBelowADInplaceOrView guard;   // outputs carry no gradient
    return f();
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// One reference to a Python object.
struct Ref {
  PyObject* o;
  explicit Ref(PyObject* p) : o(p) {
    if (!p) throw Raised{};
  }
  Ref(const Ref&) = delete;
  ~Ref() { Py_XDECREF(o); }
  PyObject* release() { return std::exchange(o, nullptr); }
};
PyObject* held(PyObject* o) {
  Py_INCREF(o);
  return o;
}
PyObject* given_or_new(PyObject* given, const at::Tensor& made) {
  return given == Py_None ? THPVariable_Wrap(made) : held(given);
}

// buf[begin : begin + n], without the dispatcher (a plan takes 6.9 us on the host so, 7.8 with a split).
at::Tensor piece(const at::Tensor& buf, int64_t begin, int64_t n) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(buf.storage()), buf.key_set(),
                                                          buf.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(begin);
  t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
  return t;
}

at::Tensor fresh(c10::IntArrayRef shape, c10::ScalarType type, const at::Device& dev) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}

// The arguments of a plan that say which rows are added.
void plan_rows(atspeed_page_plan_args& a, PyObject* add, PyObject* max_rows, PyObject* parent, int64_t B, const at::Device& dev) {
  a.max_rows = int32(max_rows, "max_rows");
  if (a.max_rows < 0) bad("max_rows must be >= 0");
  a.add = want_i32(add, "add", {B}, dev);
  if (parent == Py_None) return;
  const at::Tensor& p = tensor(parent, "parent");
  if (p.dim() != 2) bad("parent: want [B, max_nodes]");
  a.max_nodes = int32(p.size(1), "max_nodes");
  a.parent = want_i32(parent, "parent", {B, p.size(1)}, dev);
}

// held, keep, add, block_table, free_pages, n_free, page_size, max_rows, parent, stream
PyObject* page_plan(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const at::Tensor& table = gpu_tensor(o[3], "block_table");
    if (table.dim() != 2) bad("block_table: want [B, max_pages]");
    const at::Device dev = table.device();
    const int64_t B = table.size(0), most = table.size(1);
    atspeed_page_plan_args a{};
    a.B = int32(B, "B");
    a.max_pages = int32(most, "max_pages");
    a.page_size = int32(o[6], "page_size");
    plan_rows(a, o[2], o[7], o[8], B, dev);
    const int64_t R = a.max_rows, pool = tensor(o[4], "free_pages").numel();
    a.n_pool = int32(pool, "free_pages");
    a.held = want_i32(o[0], "held", {B}, dev);
    a.keep = want_i32(o[1], "keep", {B}, dev);
    a.block_table = want_i32(o[3], "block_table", {B, most}, dev);
    a.free_pages = want_i32(o[4], "free_pages", {pool}, dev);
    a.n_free = want_i32(o[5], "n_free", {1}, dev);
    at::Tensor mask;
    if (o[8] != Py_None) {
      mask = fresh({R, ((int64_t)a.max_nodes + 63) / 64}, c10::ScalarType::Long, dev);
      a.mask = address<uint64_t>(mask);
    }
    // one allocation; its pieces are the outputs
    const at::Tensor buf = fresh({4 * (B + R) + 2}, c10::ScalarType::Int, dev);
    int32_t* p = address<int32_t>(buf);
    a.n_free_out = p;
    a.length = p + 1;
    a.ctx = p + 1 + B;
    a.refused = p + 1 + 2 * B;
    a.row_off = p + 1 + 3 * B;
    p += 2 + 4 * B;
    a.row_user = p;
    a.row_pos = p + R;
    a.slot = p + 2 * R;
    a.tree_slot = p + 3 * R;
    void* const st = stream_of(o[9]);
    enqueue([&] { return atspeed_page_plan(&a, st); });
    written(o[3]);
    written(o[4]);
    Ref r(PyTuple_New(10));
    const int64_t sizes[9] = {1, B, B, B, B + 1, R, R, R, R};
    int64_t begin = 0;
    for (int i = 0; i < 9; ++i) {
      PyTuple_SET_ITEM(r.o, i, Ref(THPVariable_Wrap(piece(buf, begin, sizes[i]))).release());
      begin += sizes[i];
    }
    PyTuple_SET_ITEM(r.o, 9, mask.defined() ? Ref(THPVariable_Wrap(mask)).release() : held(Py_None));
    return r.release();
  });
}

// k, v, k_cache, v_cache, slot, stream
PyObject* kv_append(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Caches c = caches(o[2], o[3]);
    const int64_t rows = tensor(o[4], "slot").numel();
    const at::Tensor& k = rows_of(o[0], "k", rows, c.heads, c);
    const at::Tensor& v = rows_of(o[1], "v", rows, c.heads, c);
    atspeed_kv_append_args a{};
    a.dtype = c.dtype;
    a.n_rows = int32(rows, "rows");
    a.n_kv_heads = c.heads;
    a.d_head = c.dh;
    a.page_size = c.page;
    a.n_pool = c.pool;
    a.k = address<void>(k);
    a.v = address<void>(v);
    a.k_row_stride = stride(k, 0);
    a.k_head_stride = stride(k, 1);
    a.v_row_stride = stride(v, 0);
    a.v_head_stride = stride(v, 1);
    a.k_pages = c.k;
    a.v_pages = c.v;
    a.slot = want_i32(o[4], "slot", {rows}, c.dev);
    void* const st = stream_of(o[5]);
    enqueue([&] { return atspeed_kv_append(&a, st); });
    written(o[2]);
    written(o[3]);
    Py_RETURN_NONE;
  });
}

// q, k_cache, v_cache, block_table, row_off, ctx, max_ctx, max_new, mask, scale, out, return_lse, stream
PyObject* tree_attention(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const Caches c = caches(o[1], o[2]);
    const at::Tensor& q0 = tensor(o[0], "q");
    const at::Tensor& table = tensor(o[3], "block_table");
    if (q0.dim() != 3 || table.dim() != 2) bad("want q [rows, heads, d_head] and block_table [B, max_pages]");
    const int64_t rows = q0.size(0), heads = q0.size(1), B = table.size(0), most = table.size(1);
    const at::Tensor& q = rows_of(o[0], "q", rows, heads, c);
    const at::Tensor out = o[10] == Py_None ? fresh({rows, heads, c.dh}, c.type, c.dev) : rows_of(o[10], "out", rows, heads, c);
    at::Tensor lse, ws;
    atspeed_tree_attention_args a{};
    a.dtype = c.dtype;
    a.B = int32(B, "B");
    a.n_rows = int32(rows, "rows");
    a.n_heads = int32(heads, "heads");
    a.n_kv_heads = c.heads;
    a.d_head = c.dh;
    a.page_size = c.page;
    a.max_pages = int32(most, "max_pages");
    a.n_pool = c.pool;
    a.max_ctx = int32(o[6], "max_ctx");
    a.max_new = int32(o[7], "max_new");
    a.scale = o[9] == Py_None ? (float)(1.0 / std::sqrt((double)c.dh)) : number(o[9]);
    a.q = address<void>(q);
    a.q_row_stride = stride(q, 0);
    a.q_head_stride = stride(q, 1);
    a.k_pages = c.k;
    a.v_pages = c.v;
    a.block_table = want_i32(o[3], "block_table", {B, most}, c.dev);
    a.row_off = want_i32(o[4], "row_off", {B + 1}, c.dev);
    a.ctx = want_i32(o[5], "ctx", {B}, c.dev);
    if (o[8] != Py_None) {
      const at::Tensor& mask = tensor(o[8], "mask");
      if (mask.dim() != 2) bad("mask: want [rows, words]");
      a.mask_words = int32(mask.size(1), "mask words");
      a.mask = want<uint64_t>(o[8], "mask", c10::ScalarType::Long, {rows, mask.size(1)}, c.dev);
    }
    a.out = address<void>(out);
    a.out_row_stride = stride(out, 0);
    a.out_head_stride = stride(out, 1);
    const bool with_lse = flag(o[11]);
    if (with_lse) {
      lse = fresh({rows, heads}, c10::ScalarType::Float, c.dev);
      a.lse = address<float>(lse);
    }
    size_t need = 0;
    check(atspeed_tree_attention_workspace_bytes(&a, &need));
    if (need) ws = fresh({(int64_t)need}, c10::ScalarType::Byte, c.dev);
    void *const st = stream_of(o[12]), *const at = need ? address<void>(ws) : nullptr;
    enqueue([&] { return atspeed_tree_attention(&a, at, need, st); });
    written(o[10]);
    Ref result(given_or_new(o[10], out));
    if (!with_lse) return result.release();
    Ref sums(THPVariable_Wrap(lse));
    return PyTuple_Pack(2, result.o, sums.o);
  });
}

// logits, row_off, token_base, history, hist_len, repetition, frequency, presence, temperature, bias, bias_index,
// allowed, state, mask, node_token, mask_value, out, out_row, state_by_request, stream
PyObject* logit_rules(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 20, [&]() -> PyObject* {
    const at::Tensor& logits = gpu_tensor(o[0], "logits");
    if (logits.dim() != 2 || (logits.size(1) > 1 && logits.stride(1) != 1))
      bad("logits: want [rows, cols], rows contiguous");
    const at::Device dev = logits.device();
    const int64_t rows = logits.size(0), cols = logits.size(1), B = tensor(o[1], "row_off").numel() - 1;
    const c10::ScalarType f32 = c10::ScalarType::Float;
    atspeed_logit_rules_args a{};
    a.dtype = dtype_of(logits, "logits");
    a.B = int32(B, "B");
    a.n_rows = int32(rows, "rows");
    a.n_cols = int32(cols, "cols");
    a.token_base = int32(o[2], "token_base");
    at::Tensor out;
    if (o[16] == Py_None) {
      if (o[17] != Py_None) bad("out_row scatters to a given out");
      out = fresh({rows, cols}, f32, dev);
    } else {
      out = tensor(o[16], "out");
      if (out.scalar_type() != f32 || out.device() != dev || out.dim() == 0 || out.size(-1) != cols ||
          (cols > 1 && out.stride(-1) != 1))
        bad("out: want float32 [.., cols] on the logits' device, rows contiguous");
      if (out.dim() != 2) out = out.view({-1, cols});
      if (o[17] == Py_None && out.size(0) != rows) bad("out: want as many rows as logits");
    }
    a.n_out_rows = int32(out.size(0), "rows of out");
    a.mask_value = number(o[15]);
    a.logits = address<void>(logits);
    a.logits_stride = rows > 1 ? logits.stride(0) : cols;
    a.out = address<float>(out);
    a.out_stride = out.size(0) > 1 ? out.stride(0) : cols;
    a.out_row = want_i32(o[17], "out_row", {rows}, dev);
    a.row_off = want_i32(o[1], "row_off", {B + 1}, dev);
    const auto last = [](PyObject* t, const char* name) -> int64_t {
      if (t == Py_None) return 0;
      if (tensor(t, name).dim() != 2) bad(std::string(name) + ": want two dimensions");
      return tensor(t, name).size(1);
    };
    a.max_hist = int32(last(o[3], "history"), "history");
    a.history = want_i32(o[3], "history", {B, a.max_hist}, dev);
    a.hist_len = want_i32(o[4], "hist_len", {B}, dev);
    a.max_nodes = int32(last(o[14], "node_token"), "node_token");
    a.node_token = want_i32(o[14], "node_token", {B, a.max_nodes}, dev);
    a.mask_words = int32(last(o[13], "mask"), "mask");
    a.mask = want<uint64_t>(o[13], "mask", c10::ScalarType::Long, {rows, a.mask_words}, dev);
    a.repetition = want<float>(o[5], "repetition", f32, {B}, dev);
    a.frequency = want<float>(o[6], "frequency", f32, {B}, dev);
    a.presence = want<float>(o[7], "presence", f32, {B}, dev);
    a.temperature = want<float>(o[8], "temperature", f32, {B}, dev);
    if (o[9] != Py_None) {
      const at::Tensor& bias = tensor(o[9], "bias");
      if (bias.scalar_type() != f32 || bias.device() != dev || bias.dim() != 2 || bias.size(1) != cols ||
          (cols > 1 && bias.stride(1) != 1))
        bad("bias: want float32 [n, cols] on the logits' device, rows contiguous");
      a.n_bias = int32(bias.size(0), "bias");
      a.bias = address<float>(bias);
      a.bias_stride = bias.size(0) > 1 ? bias.stride(0) : cols;
    }
    a.bias_index = want_i32(o[10], "bias_index", {B}, dev);
    if (o[11] != Py_None) {
      const at::Tensor& allowed = tensor(o[11], "allowed");
      if (allowed.dim() != 2) bad("allowed: want [states, words]");
      a.n_states = int32(allowed.size(0), "allowed");
      a.allowed = reinterpret_cast<uint32_t*>(want_i32(o[11], "allowed", {allowed.size(0), (cols + 31) / 32}, dev));
    }
    a.state_by_request = flag(o[18]);
    a.state = a.state_by_request ? want_i32(o[12], "state", {B}, dev) : want_i32(o[12], "state", {rows}, dev);
    void* const st = stream_of(o[19]);
    enqueue([&] { return atspeed_logit_rules(&a, st); });
    written(o[16]);
    return given_or_new(o[16], out);
  });
}

// A float32 or bfloat16 [rows, cols] whose rows are contiguous, rows `stride` elements apart.
struct Matrix {
  const at::Tensor& t;
  int64_t rows, cols, stride;
  int32_t dtype;
};
Matrix matrix(const at::Tensor& t, const char* name) {
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) bad(std::string(name) + ": want [rows, cols], rows contiguous");
  return {t, t.size(0), t.size(1), t.size(0) > 1 ? t.stride(0) : t.size(1), dtype_of(t, name)};
}

// logits, row_off, k, score, done, token_base, log_probs, row_id, paths, path_len, stream
PyObject* beam_select(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const Matrix x = matrix(gpu_tensor(o[0], "logits"), "logits");
    const at::Device dev = x.t.device();
    const c10::ScalarType f32 = c10::ScalarType::Float, i32 = c10::ScalarType::Int;
    const int64_t B = tensor(o[1], "row_off").numel() - 1;
    atspeed_beam_select_args a{};
    a.dtype = x.dtype;
    a.B = int32(B, "B");
    a.n_rows = int32(x.rows, "rows");
    a.n_cols = int32(x.cols, "cols");
    a.k = int32(o[2], "k");
    a.token_base = int32(o[5], "token_base");
    a.log_probs = flag(o[6]);
    a.logits = address<void>(x.t);
    a.logits_stride = x.stride;
    a.row_off = want_i32(o[1], "row_off", {B + 1}, dev);
    a.score = want<float>(o[3], "score", f32, {x.rows}, dev);
    a.done = want_i32(o[4], "done", {x.rows}, dev);
    a.row_id = want_i32(o[7], "row_id", {x.rows}, dev);
    const bool with_paths = o[8] != Py_None;
    if (with_paths != (o[9] != Py_None)) bad("paths and path_len go together");
    at::Tensor empty_path;
    int64_t P = 0;
    if (with_paths) {
      const at::Tensor& paths = tensor(o[8], "paths");
      if (paths.dim() != 2 || paths.size(1) < 1) bad("paths: want [n, max_path], max_path of 1 at least");
      a.n_paths = int32(paths.size(0), "paths");
      a.max_path = int32(paths.size(1), "max_path");
      P = std::min(a.max_path, 1 << 16);   // larger ones are refused below
      a.paths = want_i32(o[8], "paths", {paths.size(0), paths.size(1)}, dev);
    }
    a.path_len = want_i32(o[9], "path_len", {a.n_paths}, dev);
    if (with_paths && a.n_paths == 0) {   // a tensor of no paths has no address: one path of no tokens is none, either
      empty_path = at::zeros({1 + P}, at::TensorOptions().dtype(i32).device(dev));
      a.n_paths = 1;
      a.path_len = address<int32_t>(empty_path);
      a.paths = a.path_len + 1;
    }
    if (B < 1 || a.k < 1) bad("want row_off of two numbers at least, and k of 1 at least");
    const int64_t k = std::min(a.k, 256);   // larger ones are refused below
    const at::Tensor count = fresh({B}, i32, dev), parent = fresh({B, k}, i32, dev), token = fresh({B, k}, i32, dev),
                     score = fresh({B, k}, f32, dev);
    at::Tensor paths, path_len, ws;
    a.count = address<int32_t>(count);
    a.parent = address<int32_t>(parent);
    a.token = address<int32_t>(token);
    a.score_out = address<float>(score);
    if (with_paths) {
      paths = fresh({B, k, P}, i32, dev);
      path_len = fresh({B, k}, i32, dev);
      a.paths_out = address<int32_t>(paths);
      a.path_len_out = address<int32_t>(path_len);
    }
    size_t need = 0;
    check(atspeed_beam_select_workspace_bytes(&a, &need));
    ws = fresh({(int64_t)need}, c10::ScalarType::Byte, dev);
    void *const st = stream_of(o[10]), *const at = address<void>(ws);
    enqueue([&] { return atspeed_beam_select(&a, at, need, st); });
    Ref r(PyTuple_New(6));
    const at::Tensor* outs[6] = {&count, &parent, &token, &score, &paths, &path_len};
    for (int i = 0; i < 6; ++i)
      PyTuple_SET_ITEM(r.o, i, outs[i]->defined() ? Ref(THPVariable_Wrap(*outs[i])).release() : held(Py_None));
    return r.release();
  });
}

// held, keep, block_table, free_pages, n_free, shared, page_size, src, stream
PyObject* page_fork(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor& table = gpu_tensor(o[2], "block_table");
    if (table.dim() != 2) bad("block_table: want [B, max_pages]");
    const at::Device dev = table.device();
    const int64_t B = table.size(0), most = table.size(1), pool = tensor(o[3], "free_pages").numel();
    atspeed_page_fork_args a{};
    a.B = int32(B, "B");
    a.page_size = int32(o[6], "page_size");
    a.max_pages = int32(most, "max_pages");
    a.n_pool = int32(pool, "free_pages");
    a.held = want_i32(o[0], "held", {B}, dev);
    a.keep = want_i32(o[1], "keep", {B}, dev);
    a.src = want_i32(o[7], "src", {B}, dev);
    a.block_table = want_i32(o[2], "block_table", {B, most}, dev);
    a.free_pages = want_i32(o[3], "free_pages", {pool}, dev);
    a.n_free = want_i32(o[4], "n_free", {1}, dev);
    a.shared = want_i32(o[5], "shared", {pool}, dev);
    const at::Tensor buf = fresh({5 * B}, c10::ScalarType::Int, dev);
    int32_t* p = address<int32_t>(buf);
    a.length = p;
    a.refused = p + B;
    a.copy_src = p + 2 * B;
    a.copy_dst = p + 3 * B;
    a.copy_len = p + 4 * B;
    size_t need = 0;
    check(atspeed_page_fork_workspace_bytes(&a, &need));
    const at::Tensor ws = fresh({(int64_t)need}, c10::ScalarType::Byte, dev);
    void *const st = stream_of(o[8]), *const at = address<void>(ws);
    enqueue([&] { return atspeed_page_fork(&a, at, need, st); });
    for (const int i : {2, 3, 4, 5}) written(o[i]);
    Ref r(PyTuple_New(5));
    for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(r.o, i, Ref(THPVariable_Wrap(piece(buf, i * B, B))).release());
    return r.release();
  });
}

// Caches of one layer [pages, page_size, kv_heads, d_head] or several [layers, ...].
struct Layers {
  Caches c;
  int32_t n;
  int64_t k_stride, v_stride;
};
Layers layers(PyObject* ko, PyObject* vo) {
  const at::Tensor& k = gpu_tensor(ko, "k_cache");
  const at::Tensor& v = tensor(vo, "v_cache");
  if (k.dim() == 4) return {caches(ko, vo), 1, 0, 0};
  if (k.dim() != 5) bad("k_cache: want [layers, pages, page_size, kv_heads, d_head]");
  if (v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type() || v.device() != k.device() || k.stride(4) != 1 ||
      v.stride(4) != 1)
    bad("the caches want one type, shape and device, the last dimension contiguous");
  return {{k.device(), k.scalar_type(), dtype_of(k, "k_cache"), int32(k.size(1), "pages"), int32(k.size(2), "page_size"),
           int32(k.size(3), "kv_heads"), int32(k.size(4), "d_head"),
           {address<void>(k), stride(k, 1), stride(k, 2), stride(k, 3)},
           {address<void>(v), stride(v, 1), stride(v, 2), stride(v, 3)}},
          int32(k.size(0), "layers"), stride(k, 0), stride(v, 0)};
}
template <class A>
void set_layers(A& a, const Layers& l) {
  a.dtype = l.c.dtype;
  a.n_layers = l.n;
  a.n_kv_heads = l.c.heads;
  a.d_head = l.c.dh;
  a.page_size = l.c.page;
  a.n_pool = l.c.pool;
  a.k_pages = l.c.k;
  a.v_pages = l.c.v;
  a.k_layer_stride = l.k_stride;
  a.v_layer_stride = l.v_stride;
}

// add, block_table, max_rows, parent, k_cache, v_cache: what page_copy and page_plan will look at behind a fork, which
// changes the tables.  Launches nothing.
PyObject* fork_check(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const at::Tensor& table = gpu_tensor(o[1], "block_table");
    if (table.dim() != 2) bad("block_table: want [B, max_pages]");
    atspeed_page_plan_args a{};
    plan_rows(a, o[0], o[2], o[3], table.size(0), table.device());
    if (!a.add && table.size(0) > 0) bad("add: want a tensor");
    if (o[3] != Py_None && (a.max_nodes < 1 || a.max_nodes > 4096)) bad("parent: want [B, max_nodes], max_nodes 1..4096");
    const Layers l = layers(o[4], o[5]);
    if (l.c.dev != table.device()) bad("the caches and the block_table want one device");
    atspeed_page_copy_args c{};
    set_layers(c, l);
    check(atspeed_page_copy(&c, nullptr));   // of no pages
    Py_RETURN_NONE;
  });
}

// k_cache, v_cache, src, dst, length, stream
PyObject* page_copy(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Layers l = layers(o[0], o[1]);
    const int64_t rows = tensor(o[2], "src").numel();
    atspeed_page_copy_args a{};
    set_layers(a, l);
    a.n = int32(rows, "copies");
    a.src = want_i32(o[2], "src", {rows}, l.c.dev);
    a.dst = want_i32(o[3], "dst", {rows}, l.c.dev);
    a.length = want_i32(o[4], "length", {rows}, l.c.dev);
    void* const st = stream_of(o[5]);
    enqueue([&] { return atspeed_page_copy(&a, st); });
    written(o[0]);
    written(o[1]);
    Py_RETURN_NONE;
  });
}

// k_cache, v_cache, block_table, ctx, path, n_path, length, stream
PyObject* kv_compact(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Layers l = layers(o[0], o[1]);
    const at::Tensor& table = tensor(o[2], "block_table");
    const at::Tensor& path = tensor(o[4], "path");
    if (table.dim() != 2 || path.dim() != 2) bad("want block_table [B, max_pages] and path [B, max_path]");
    const int64_t B = table.size(0), most = table.size(1), P = path.size(1);
    atspeed_kv_compact_args a{};
    set_layers(a, l);
    a.B = int32(B, "B");
    a.max_pages = int32(most, "max_pages");
    a.max_path = int32(P, "max_path");
    a.block_table = want_i32(o[2], "block_table", {B, most}, l.c.dev);
    a.ctx = want_i32(o[3], "ctx", {B}, l.c.dev);
    a.path = want_i32(o[4], "path", {B, P}, l.c.dev);
    a.n_path = want_i32(o[5], "n_path", {B}, l.c.dev);
    const int32_t* const length = want_i32(o[6], "length", {B}, l.c.dev);
    at::Tensor keep;
    if (length) keep = fresh({B}, c10::ScalarType::Int, l.c.dev);
    int32_t* const to = length ? address<int32_t>(keep) : nullptr;
    void* const st = stream_of(o[7]);
    enqueue([&] { return length ? atspeed_kv_compact_keep(&a, length, to, st) : atspeed_kv_compact(&a, st); });
    written(o[0]);
    written(o[1]);
    if (length) return THPVariable_Wrap(keep);
    Py_RETURN_NONE;
  });
}

// logits, teacher_logit, teacher_index, tail, weight, temperature, reverse, stream
PyObject* distill_loss(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Matrix x = matrix(gpu_tensor(o[0], "logits"), "logits");
    const at::Device dev = x.t.device();
    const c10::ScalarType f32 = c10::ScalarType::Float;
    const at::Tensor& index = tensor(o[2], "teacher_index");
    if (index.dim() != 2) bad("teacher_index: want [rows, tops]");
    const int64_t m = index.size(1);
    atspeed_distill_loss_args a{};
    a.dtype = x.dtype;
    a.n_rows = int32(x.rows, "rows");
    a.n_cols = int32(x.cols, "cols");
    a.n_tops = int32(m, "tops");
    a.reverse = flag(o[6]);
    a.temperature = number(o[5]);
    a.logits = address<void>(x.t);
    a.logits_stride = x.stride;
    tensor(o[1], "teacher_logit");
    a.teacher_logit = want<void>(o[1], "teacher_logit", x.t.scalar_type(), {x.rows, m}, dev);
    a.teacher_index = want_i32(o[2], "teacher_index", {x.rows, m}, dev);
    a.tail = want<float>(o[3], "tail", f32, {x.rows}, dev);
    a.weight = want<float>(o[4], "weight", f32, {x.rows}, dev);
    const at::Tensor loss = fresh({x.rows}, f32, dev), saved = fresh({x.rows, 2 + m}, f32, dev);
    a.loss = address<float>(loss);
    a.saved = address<float>(saved);
    void* const st = stream_of(o[7]);
    enqueue([&] { return atspeed_distill_loss(&a, st); });
    Ref r(PyTuple_New(2));
    PyTuple_SET_ITEM(r.o, 0, Ref(THPVariable_Wrap(loss)).release());
    PyTuple_SET_ITEM(r.o, 1, Ref(THPVariable_Wrap(saved)).release());
    return r.release();
  });
}

// logits, teacher_index, saved, grad_loss, temperature, out, stream
PyObject* distill_grad(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const Matrix x = matrix(gpu_tensor(o[0], "logits"), "logits");
    const at::Device dev = x.t.device();
    const c10::ScalarType f32 = c10::ScalarType::Float;
    const at::Tensor& index = tensor(o[1], "teacher_index");
    if (index.dim() != 2) bad("teacher_index: want [rows, tops]");
    const int64_t m = index.size(1);
    const at::Tensor out = o[5] == Py_None ? fresh({x.rows, x.cols}, x.t.scalar_type(), dev) : tensor(o[5], "out");
    const Matrix g = matrix(out, "out");
    if (g.rows != x.rows || g.cols != x.cols || g.dtype != x.dtype || out.device() != dev)
      bad("out: want the logits' type, shape and device");
    atspeed_distill_grad_args a{};
    a.dtype = x.dtype;
    a.n_rows = int32(x.rows, "rows");
    a.n_cols = int32(x.cols, "cols");
    a.n_tops = int32(m, "tops");
    a.temperature = number(o[4]);
    a.logits = address<void>(x.t);
    a.logits_stride = x.stride;
    a.teacher_index = want_i32(o[1], "teacher_index", {x.rows, m}, dev);
    tensor(o[2], "saved");
    a.saved = want<float>(o[2], "saved", f32, {x.rows, 2 + m}, dev);
    a.grad_loss = want<float>(o[3], "grad_loss", f32, {x.rows}, dev);
    a.grad = address<void>(out);
    a.grad_stride = g.stride;
    void* const st = stream_of(o[6]);
    enqueue([&] { return atspeed_distill_grad(&a, st); });
    written(o[5]);
    return given_or_new(o[5], out);
  });
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_XINCREF(cls);
  Py_XSETREF(g_error, cls);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(page_plan), FAST(kv_append), FAST(tree_attention), FAST(logit_rules),
                         FAST(beam_select), FAST(page_fork), FAST(fork_check), FAST(page_copy), FAST(kv_compact), FAST(distill_loss),
                         FAST(distill_grad),
                         {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
