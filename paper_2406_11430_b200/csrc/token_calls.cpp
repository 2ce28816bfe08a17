// Argument marshalling of the calls on packed new tokens, for the Python binding.  The smallest of these calls
// run 3 us on the GPU; describing a dozen tensors through ctypes took 10 to 15 us more on the host.  This module
// does what the ctypes wrappers of the other calls do -- check that tensors fit together (ValueError), fill in
// the C structures, call the library -- and returns the library's status.  The entry points are handed over
// as addresses, so whichever build of the library the binding has loaded is the one that is called.
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "l2kv.h"

namespace {

struct Bad { std::string what; };                        // becomes a ValueError

decltype(&l2kv_rotary_write) fn_rotary_write;
decltype(&l2kv_tree_commit) fn_tree_commit;
decltype(&l2kv_prompt_attention) fn_prompt_attention;
decltype(&l2kv_tree_attention) fn_tree_attention;
decltype(&l2kv_prompt_attention_workspace_bytes) fn_workspace_bytes;

// A tensor argument; null for None.
const at::Tensor* tensor(PyObject* o, const char* what, bool may_be_none = false) {
  if (o == Py_None && may_be_none) return nullptr;
  if (!THPVariable_Check(o)) throw Bad{std::string(what) + " is not a tensor"};
  return &THPVariable_Unpack(o);
}
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Bad{""};
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Bad{""};
  return v;
}
// What is an int32 of the library's: a size, or an argument.
int32_t narrow(int64_t v, const char* what) {
  if (v != (int32_t)v) throw Bad{std::string(what) + " is out of range"};
  return (int32_t)v;
}
int32_t integer32(PyObject* o, const char* what) { return narrow(integer(o), what); }
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Bad{""};
  return v != 0;
}

int dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return L2KV_BF16;
  if (t.scalar_type() == at::kFloat) return L2KV_F32;
  throw Bad{"unsupported dtype " + std::string(c10::toString(t.scalar_type()))};
}

void entries(const at::Tensor* t, int64_t count, const char* what, at::ScalarType type = at::kInt) {
  if (t && (t->scalar_type() != type || !t->is_contiguous() || (count >= 0 && t->numel() != count)))
    throw Bad{std::string(what) + " must be contiguous " + c10::toString(type) +
              (count >= 0 ? " with " + std::to_string(count) + " entries" : "")};
}

struct Attr {                                            // an attribute of the rows object, held while this lives
  PyObject* o = nullptr;
  Attr() = default;
  Attr(PyObject* of, const char* name) { get(of, name); }
  Attr(const Attr&) = delete;
  ~Attr() { Py_XDECREF(o); }
  void get(PyObject* of, const char* name) { if (!(o = PyObject_GetAttrString(of, name))) throw Bad{""}; }
};
// The row ranges of a packed cache, held for a call: other threads run meanwhile.
struct Ranges { Attr off, cap; };

// A call of the library.  Other Python threads run while it lasts: it can block for as long as the GPU's queue is full.
// (The arguments are worked out before, and the caller holds the tensors.)
template <typename... P, typename... A>
PyObject* unlocked(int (*fn)(P...), A... args) {
  PyThreadState* const state = PyEval_SaveThread();
  const int rc = fn(args...);
  PyEval_RestoreThread(state);
  return PyLong_FromLong(rc);
}

// Geometry of a cache, as the binding's Layout takes it from a tensor.
l2kv_layout layout(const at::Tensor& K, int64_t q_heads, PyObject* rows, Ranges* held) {
  l2kv_layout a{};
  a.dtype = dtype_of(K);
  a.q_heads = narrow(q_heads, "the number of query heads");
  if (rows != Py_None) {
    held->off.get(rows, "off");
    held->cap.get(rows, "cap");
    const Attr B(rows, "B"), L(rows, "L"), t_cap(rows, "t_cap"), total(rows, "total_rows");
    a.total_rows = integer(total.o);
    if (K.dim() != 3 || K.stride(2) != 1 || K.size(1) != a.total_rows)
      throw Bad{"packed cache must be [Hkv, total_rows, D] with D contiguous"};
    const at::Tensor *o = tensor(held->off.o, "rows.off"), *c = tensor(held->cap.o, "rows.cap");
    if (o->device() != K.device() || c->device() != K.device()) throw Bad{"rows on another device than the cache"};
    a.batch = integer32(B.o, "rows.B"); a.layers = integer32(L.o, "rows.L"); a.t_cap = integer32(t_cap.o, "rows.t_cap");
    // the kernels read these as int64 and int32 arrays and write where they say
    entries(o, (int64_t)a.batch * a.layers, "rows.off", at::kLong);
    entries(c, (int64_t)a.batch * a.layers, "rows.cap");
    a.kv_heads = narrow(K.size(0), "a cache's size"); a.head_dim = narrow(K.size(2), "a cache's size");
    a.stride_h = K.stride(0); a.stride_t = K.stride(1);
    a.row_off_dev = static_cast<const int64_t*>(o->data_ptr());
    a.row_cap_dev = static_cast<const int32_t*>(c->data_ptr());
    return a;
  }
  if (K.dim() != 5 || K.stride(4) != 1) throw Bad{"cache must be [B, L, Hkv, t_cap, D] with D contiguous"};
  int32_t* const sizes[5] = {&a.batch, &a.layers, &a.kv_heads, &a.t_cap, &a.head_dim};
  for (int i = 0; i < 5; ++i) *sizes[i] = narrow(K.size(i), "a cache's size");
  a.stride_b = K.stride(0); a.stride_l = K.stride(1); a.stride_h = K.stride(2); a.stride_t = K.stride(3);
  return a;
}

// Every tensor of a call lies where the cache lies: kernels run on one device.
template <typename... T>
void one_device(const at::Tensor& ref, const T*... ts) {
  for (const at::Tensor* t : {static_cast<const at::Tensor*>(ts)...})
    if (t && t->device() != ref.device())
      throw Bad{"a tensor on " + t->device().str() + " in a call on " + ref.device().str()};
}

// Host tensors are checked like others, but no kernel may see them.
uint32_t flags_of(const at::Tensor& K, bool per_head) {
  return (per_head ? L2KV_TOKENS_LEN_PER_HEAD : 0) | (K.is_cuda() ? 0 : L2KV_TOKENS_NO_LAUNCH);
}

// V has K's geometry: one set of strides describes both.
void same_geometry(const at::Tensor& K, const at::Tensor* V) {
  if (V && (V->scalar_type() != K.scalar_type() || V->sizes() != K.sizes() || V->strides() != K.strides()))
    throw Bad{"V must have the dtype, shape and strides of K"};
}

int64_t heads_of(const at::Tensor& t) {
  if (t.dim() != 3 && t.dim() != 4) throw Bad{"tokens must be [L, N, heads, D] (or [N, heads, D] for one layer)"};
  return t.size(-2);
}

// Rows of new tokens: [L, N, heads, D], or [N, heads, D] where L is 1.
l2kv_tokens tokens(const at::Tensor& t, const l2kv_layout& a, int64_t n, int64_t heads) {
  const int d = (int)t.dim();
  if ((d != 3 && d != 4) || t.stride(d - 1) != 1 || (d == 4 ? t.size(0) : 1) != a.layers || t.size(d - 1) != a.head_dim)
    throw Bad{"tokens must be [L, N, heads, D] (or [N, heads, D] for one layer) with D contiguous"};
  if (dtype_of(t) != a.dtype) throw Bad{"tokens do not have the cache's dtype"};
  if (t.size(d - 3) != n || t.size(d - 2) != heads) throw Bad{"tokens differ in number or heads"};
  return {t.data_ptr(), d == 4 ? t.stride(0) : 0, t.stride(d - 3), t.stride(d - 2)};
}

int64_t n_lengths(const l2kv_layout& a, bool per_head) { return (int64_t)a.batch * a.layers * (per_head ? a.kv_heads : 1); }
// What lies along the cache's rows: one entry per row and head (-1, any number, for a cache without rows).
int64_t n_rows(const l2kv_layout& a) {
  const int64_t n = a.row_off_dev ? (int64_t)a.kv_heads * a.total_rows : (int64_t)a.batch * a.layers * a.kv_heads * a.t_cap;
  return n > 0 ? n : -1;
}

void check_count(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) throw Bad{"wrong number of arguments"};
}

template <typename F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Bad& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what.c_str());
  } catch (const std::exception& e) {                    // e.g. a tensor without storage
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
  }
  return nullptr;
}

PyObject* rotary_write(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject* {
    check_count(n_args, 19);
    const at::Tensor *q = tensor(v[0], "q", true), *k = tensor(v[1], "k"), *val = tensor(v[2], "v"),
                     *off = tensor(v[3], "tok_off"), *pos = tensor(v[4], "pos", true), *freq = tensor(v[5], "freq", true),
                     *q_out = tensor(v[6], "q_out", true), *K = tensor(v[7], "K_c"), *V = tensor(v[8], "V_c", true),
                     *idx = tensor(v[9], "idx", true), *key = tensor(v[10], "sumsq_c", true),
                     *start = tensor(v[11], "start_dev"), *cur = tensor(v[12], "cur_len_dev"), *ws = tensor(v[13], "workspace");
    const bool interleaved = truth(v[14]), per_head = truth(v[17]);
    Ranges held;
    const l2kv_layout a = layout(*K, q ? heads_of(*q) : 0, v[16], &held);
    one_device(*K, q, k, val, off, pos, freq, q_out, V, idx, key, start, cur, ws);
    same_geometry(*K, V);
    heads_of(*k);
    const int32_t n = narrow(k->size(-3), "the number of tokens");
    entries(off, (int64_t)a.batch + 1, "tok_off");
    entries(pos, n, "pos");
    entries(freq, -1, "freq", at::kDouble);
    entries(idx, n_rows(a), "idx");
    entries(key, n_rows(a), "sumsq_c", at::kFloat);
    entries(start, n_lengths(a, per_head), "start_dev");
    entries(cur, n_lengths(a, per_head), "cur_len_dev");
    entries(ws, -1, "workspace", at::kByte);
    l2kv_tokens tq{}, to{};
    if (q) tq = tokens(*q, a, n, a.q_heads);
    if (q_out) to = tokens(*q_out, a, n, a.q_heads);
    const l2kv_tokens tk = tokens(*k, a, n, a.kv_heads), tv = tokens(*val, a, n, a.kv_heads);
    return unlocked(fn_rotary_write,
        q ? &tq : nullptr, &tk, &tv, static_cast<const int32_t*>(ptr(off)), n, static_cast<const int32_t*>(ptr(pos)),
        static_cast<const double*>(ptr(freq)), freq ? narrow(2 * freq->numel(), "the number of frequencies") : 0,
        real(v[15]), q_out ? &to : nullptr, ptr(K), ptr(V), static_cast<int32_t*>(ptr(idx)), static_cast<float*>(ptr(key)), &a,
        static_cast<const int32_t*>(ptr(start)), static_cast<int32_t*>(ptr(cur)),
        flags_of(*K, per_head) | (interleaved ? L2KV_TOKENS_ROTARY_INTERLEAVED : 0), ptr(ws),
        (size_t)ws->numel(), reinterpret_cast<void*>(integer(v[18])));
  });
}

PyObject* tree_commit(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject* {
    check_count(n_args, 13);
    const at::Tensor *K = tensor(v[0], "K_c"), *V = tensor(v[1], "V_c", true), *idx = tensor(v[2], "idx", true),
                     *key = tensor(v[3], "sumsq_c", true), *start = tensor(v[4], "start_dev"), *cur = tensor(v[5], "cur_len_dev"),
                     *path = tensor(v[6], "path"), *n_path = tensor(v[7], "n_path"), *out = tensor(v[8], "len_out_dev"),
                     *ws = tensor(v[9], "workspace");
    const bool per_head = truth(v[11]);
    Ranges held;
    const l2kv_layout a = layout(*K, K->dim() > 2 ? K->size(v[10] != Py_None ? 0 : 2) : 0, v[10], &held);
    if (path->dim() != 2 || path->size(0) != a.batch) throw Bad{"path must be [B, path_cap]"};
    one_device(*K, V, idx, key, start, cur, path, n_path, out, ws);
    same_geometry(*K, V);
    entries(path, -1, "path");
    entries(n_path, a.batch, "n_path");
    entries(idx, n_rows(a), "idx");
    entries(key, n_rows(a), "sumsq_c", at::kFloat);
    entries(start, n_lengths(a, per_head), "start_dev");
    entries(cur, n_lengths(a, per_head), "cur_len_dev");
    entries(out, n_lengths(a, per_head), "len_out_dev");
    entries(ws, -1, "workspace", at::kByte);
    return unlocked(fn_tree_commit,
        ptr(K), ptr(V), static_cast<int32_t*>(ptr(idx)), static_cast<float*>(ptr(key)), &a,
        static_cast<const int32_t*>(ptr(start)), static_cast<const int32_t*>(ptr(cur)), static_cast<const int32_t*>(ptr(path)),
        narrow(path->size(1), "the length of a path"), static_cast<const int32_t*>(ptr(n_path)), static_cast<int32_t*>(ptr(out)),
        flags_of(*K, per_head), ptr(ws), (size_t)ws->numel(), reinterpret_cast<void*>(integer(v[12])));
  });
}

PyObject* attention(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject* {
    check_count(n_args, 14);
    const at::Tensor *q = tensor(v[0], "q"), *off = tensor(v[1], "tok_off"), *mask = tensor(v[2], "tree_mask", true),
                     *K = tensor(v[3], "K_c"), *V = tensor(v[4], "V_c", true), *cur = tensor(v[5], "cur_len_dev"),
                     *out = tensor(v[7], "out"), *lse = tensor(v[8], "lse_out", true), *ws = tensor(v[10], "workspace", true);
    const bool per_head = truth(v[12]);
    Ranges held;
    const l2kv_layout a = layout(*K, heads_of(*q), v[11], &held);
    const int32_t n = narrow(q->size(-3), "the number of tokens");
    one_device(*K, q, off, mask, V, cur, out, lse, ws);
    same_geometry(*K, V);
    entries(off, (int64_t)a.batch + 1, "tok_off");
    entries(cur, n_lengths(a, per_head), "cur_len_dev");
    entries(lse, (int64_t)a.layers * n * a.q_heads, "lse_out", at::kFloat);
    entries(ws, -1, "workspace", at::kByte);
    const l2kv_tokens tq = tokens(*q, a, n, a.q_heads), to = tokens(*out, a, n, a.q_heads);
    void* stream = reinterpret_cast<void*>(integer(v[13]));
    const int32_t max_len = integer32(v[6], "max_len");
    const float scale = (float)real(v[9]);
    const uint32_t flags = flags_of(*K, per_head);
    const size_t ws_bytes = ws ? (size_t)ws->numel() : 0;
    if (!mask)
      return unlocked(fn_prompt_attention,
          &tq, static_cast<const int32_t*>(ptr(off)), n, ptr(K), ptr(V), &a, static_cast<const int32_t*>(ptr(cur)),
          max_len, scale, flags, &to, static_cast<float*>(ptr(lse)), ptr(ws), ws_bytes, stream);
    if (mask->dim() != 2 || mask->size(0) != n || (mask->scalar_type() != at::kLong && mask->scalar_type() != at::kUInt64) ||
        !mask->is_contiguous())
      throw Bad{"tree_mask must be contiguous int64 or uint64 [N, words]"};
    return unlocked(fn_tree_attention,
        &tq, static_cast<const int32_t*>(ptr(off)), n, static_cast<const uint64_t*>(ptr(mask)), narrow(mask->size(1), "the words of a mask"),
        ptr(K), ptr(V), &a, static_cast<const int32_t*>(ptr(cur)), max_len, scale, flags, &to, static_cast<float*>(ptr(lse)),
        ptr(ws), ws_bytes, stream);
  });
}

// (K_c, q, max_len, rows) -> bytes, or a negative status
PyObject* workspace_bytes(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject* {
    check_count(n_args, 4);
    const at::Tensor *K = tensor(v[0], "K_c"), *q = tensor(v[1], "q");
    Ranges held;
    const l2kv_layout a = layout(*K, heads_of(*q), v[3], &held);
    size_t bytes = 0;
    const int rc = fn_workspace_bytes(&a, narrow(q->size(-3), "the number of tokens"), integer32(v[2], "max_len"), &bytes);
    return PyLong_FromLongLong(rc == L2KV_OK ? (long long)bytes : rc);
  });
}

// The addresses of the library's entry points, in the order below.
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  return guarded([&]() -> PyObject* {
    check_count(n_args, 5);
    auto at = [&](int i) { return reinterpret_cast<void*>(integer(v[i])); };
    fn_rotary_write = reinterpret_cast<decltype(fn_rotary_write)>(at(0));
    fn_tree_commit = reinterpret_cast<decltype(fn_tree_commit)>(at(1));
    fn_prompt_attention = reinterpret_cast<decltype(fn_prompt_attention)>(at(2));
    fn_tree_attention = reinterpret_cast<decltype(fn_tree_attention)>(at(3));
    fn_workspace_bytes = reinterpret_cast<decltype(fn_workspace_bytes)>(at(4));
    Py_RETURN_NONE;
  });
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
    {"rotary_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary_write)), METH_FASTCALL, nullptr},
    {"tree_commit", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(tree_commit)), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attention)), METH_FASTCALL, nullptr},
    {"workspace_bytes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(workspace_bytes)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_token_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__token_calls() { return PyModule_Create(&module_def); }
