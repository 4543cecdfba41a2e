// The ordinary call of the entry points, without ctypes: plain CUDA tensors on the current device and its current
// stream, default parameters.  The checks are those of binding.py; whatever is not ordinary (another type, device, layout or argument)
// returns None, and binding.py takes its general path, which says what is wrong.  A call takes 0.5 us here, 2 to 2.6 through ctypes
// (six attribute reads and conversions a tensor), where the launch itself takes 3 and the smallest kernels 3 to 4.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <limits>
#include <utility>

#include "../../include/swz.h"
#include "../../include/swz_attention.h"

namespace {

using GemmFn = decltype(&swz_gemm);
using TransposeFn = decltype(&swz_transpose);
using SoftmaxFn = decltype(&swz_softmax);
using LayernormFn = decltype(&swz_layernorm);
GemmFn g_gemm;
TransposeFn g_transpose;
SoftmaxFn g_softmax;
LayernormFn g_layernorm;
PyObject* g_parameter;         // torch.nn.Parameter

// A torch.Tensor or Parameter (no other subclass) with memory on `device`, contiguous; nullptr otherwise.
const at::Tensor* plain(PyObject* o, c10::DeviceIndex device) {
  PyObject* type = reinterpret_cast<PyObject*>(Py_TYPE(o));
  if (type != THPVariableClass && type != g_parameter) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.get_device() != device || t.layout() != at::kStrided || !t.has_storage() || !t.is_contiguous()) return nullptr;
  return &t;
}

bool is_bf16(const at::Tensor* t, int dim) { return t != nullptr && t->dim() == dim && t->scalar_type() == at::kBFloat16; }

bool as_int(PyObject* o, int* out) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow != 0 || v < std::numeric_limits<int>::min() || v > std::numeric_limits<int>::max()) return false;
  *out = static_cast<int>(v);
  return true;
}

// call(stream) without the interpreter lock, as ctypes does it; its status as a Python integer
template <class F>
PyObject* launch(c10::DeviceIndex device, F&& call) {
  const hipStream_t stream = c10::hip::getCurrentHIPStream(device).stream();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call(stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// C++ exceptions of the tensor library (a tensor that refuses its pointer, say) go to the general path too
template <class F>
PyObject* guarded(F&& body) {
  try {
    PyObject* r = body();
    if (r != nullptr) return r;
  } catch (...) {
  }
  Py_RETURN_NONE;
}

PyObject* gemm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int mode;
    if (n != 4 || !as_int(args[3], &mode)) return nullptr;
    const c10::DeviceIndex dev = c10::hip::current_device();
    const at::Tensor *a = plain(args[0], dev), *b = plain(args[1], dev), *c = plain(args[2], dev);
    if (!is_bf16(a, 2) || !is_bf16(b, 2) || !is_bf16(c, 2)) return nullptr;
    const int64_t M = a->size(0), K = a->size(1), N = b->size(1);
    if (b->size(0) != K || c->size(0) != M || c->size(1) != N) return nullptr;
    void *pa = a->data_ptr(), *pb = b->data_ptr(), *pc = c->data_ptr();
    return launch(dev, [&](hipStream_t s) { return g_gemm(pa, pb, pc, M, N, K, SWZ_DTYPE_BF16, mode, s); });
  });
}

PyObject* transpose(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int tile, mode;
    if (n != 4 || !as_int(args[2], &tile) || !as_int(args[3], &mode)) return nullptr;
    const c10::DeviceIndex dev = c10::hip::current_device();
    const at::Tensor *x = plain(args[0], dev), *out = plain(args[1], dev);
    if (x == nullptr || out == nullptr || x->dim() != 2 || out->dim() != 2 || x->scalar_type() != out->scalar_type()) return nullptr;
    const int64_t M = x->size(0), N = x->size(1), bytes = static_cast<int64_t>(x->element_size());
    if (out->size(0) != N || out->size(1) != M || (bytes != 2 && bytes != 4)) return nullptr;
    void *px = x->data_ptr(), *po = out->data_ptr();
    return launch(dev, [&](hipStream_t s) { return g_transpose(px, po, M, N, static_cast<int>(bytes), tile, mode, nullptr, s); });
  });
}

PyObject* softmax(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int chunks, mode;
    if (n != 4 || !as_int(args[2], &chunks) || !as_int(args[3], &mode)) return nullptr;
    const c10::DeviceIndex dev = c10::hip::current_device();
    const at::Tensor *x = plain(args[0], dev), *out = plain(args[1], dev);
    if (!is_bf16(x, 2) || !is_bf16(out, 2) || x->sizes() != out->sizes()) return nullptr;
    const int64_t M = x->size(0), N = x->size(1);
    void *px = x->data_ptr(), *po = out->data_ptr();
    return launch(dev, [&](hipStream_t s) { return g_softmax(px, po, M, N, chunks, mode, nullptr, s); });
  });
}

PyObject* layernorm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int chunks, mode;
    if (n != 7 || !PyFloat_CheckExact(args[4]) || !as_int(args[5], &chunks) || !as_int(args[6], &mode)) return nullptr;
    const float eps = static_cast<float>(PyFloat_AS_DOUBLE(args[4]));
    const c10::DeviceIndex dev = c10::hip::current_device();
    const at::Tensor *x = plain(args[0], dev), *g = plain(args[1], dev), *b = plain(args[2], dev), *out = plain(args[3], dev);
    if (!is_bf16(x, 2) || !is_bf16(out, 2) || !is_bf16(g, 1) || !is_bf16(b, 1) || x->sizes() != out->sizes()) return nullptr;
    const int64_t M = x->size(0), N = x->size(1);
    if (g->size(0) != N || b->size(0) != N) return nullptr;
    void *px = x->data_ptr(), *pg = g->data_ptr(), *pb = b->data_ptr(), *po = out->data_ptr();
    return launch(dev, [&](hipStream_t s) { return g_layernorm(px, pg, pb, po, M, N, eps, chunks, mode, nullptr, s); });
  });
}

// ---------------------------------------------------------------- attention layers (include/swz_attention.h, attention_layer.py)
// Outputs and workspaces are made here; what is returned is the result, the status of a call that failed (an integer), or None for the general path.

struct AttentionFns {
  decltype(&swz_qk_norm_rope) norm;
  decltype(&swz_qk_norm_rope_backward_workspace) norm_backward_workspace;
  decltype(&swz_qk_norm_rope_backward) norm_backward;
  decltype(&swz_attention_workspace) attention_workspace;
  decltype(&swz_attention) attention;
  decltype(&swz_attention_backward_workspace) attention_backward_workspace;
  decltype(&swz_attention_backward) attention_backward;
  decltype(&swz_cache4_append) append;
  decltype(&swz_cache4_read) read;
  decltype(&swz_cache4_attention_workspace) cache_attention_workspace;
  decltype(&swz_cache4_attention) cache_attention;
} g_attention;

// As `plain`, of any strides.
const at::Tensor* on_device(PyObject* o, c10::DeviceIndex device) {
  PyObject* type = reinterpret_cast<PyObject*>(Py_TYPE(o));
  if (type != THPVariableClass && type != g_parameter) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}

bool is_heads(const at::Tensor* t) { return t != nullptr && t->dim() == 3 && t->scalar_type() == at::kBFloat16 && t->stride(2) == 1 && t->numel() > 0; }
bool is_type(const at::Tensor* t, int dim, at::ScalarType type) { return t != nullptr && t->dim() == dim && t->scalar_type() == type; }
bool is_ints(const at::Tensor* t, int64_t n) { return is_type(t, 1, at::kInt) && t->size(0) == n; }

swz_heads heads_of(const at::Tensor& t) { return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0}; }
at::Tensor dense_like(const at::Tensor& t) { return at::empty(t.sizes(), t.options()); }
at::Tensor workspace(int64_t bytes, const at::Tensor& like) { return at::empty({bytes}, like.options().dtype(at::kByte)); }

bool as_float(PyObject* o, float* out) {
  if (!PyFloat_CheckExact(o)) return false;
  *out = static_cast<float>(PyFloat_AS_DOUBLE(o));
  return true;
}

PyObject* tuple_of(std::initializer_list<at::Tensor> tensors) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(tensors.size()));
  Py_ssize_t i = 0;
  if (r != nullptr)
    for (const at::Tensor& t : tensors) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
  return r;
}

// The status of call(stream) where it is not 0, else what `result` makes.
template <class F, class R>
PyObject* result_of(c10::DeviceIndex device, F&& call, R&& result) {
  const hipStream_t stream = c10::hip::getCurrentHIPStream(device).stream();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call(stream);
  Py_END_ALLOW_THREADS
  return status != 0 ? PyLong_FromLong(status) : result();
}

// args: q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved
struct NormCall {
  const at::Tensor *q, *k;
  swz_norm_args a;
};
bool norm_call(PyObject* const* args, c10::DeviceIndex dev, NormCall* c) {
  c->q = on_device(args[0], dev), c->k = on_device(args[1], dev);
  const at::Tensor *wq = plain(args[2], dev), *wk = plain(args[3], dev), *cos = plain(args[4], dev), *sin = plain(args[5], dev), *p = plain(args[6], dev);
  float eps;
  if (!is_heads(c->q) || !is_heads(c->k) || !is_bf16(wq, 1) || !is_bf16(wk, 1) || !is_type(cos, 2, at::kFloat) || !is_type(sin, 2, at::kFloat)) return false;
  const int64_t tokens = c->q->size(0), dim = c->q->size(2);
  if (c->k->size(0) != tokens || c->k->size(2) != dim || wq->size(0) != dim || wk->size(0) != dim || cos->sizes() != sin->sizes() || !is_ints(p, tokens)) return false;
  if (!as_float(args[7], &eps) || !PyBool_Check(args[8]) || c->q->size(1) > 65536 || c->k->size(1) > 65536 || cos->size(1) > 1024) return false;
  c->a = {heads_of(*c->q), heads_of(*c->k), {}, {}, wq->data_ptr(), wk->data_ptr(), static_cast<const float*>(cos->data_ptr()), static_cast<const float*>(sin->data_ptr()),
          static_cast<const int32_t*>(p->data_ptr()), tokens, static_cast<int32_t>(c->q->size(1)), static_cast<int32_t>(c->k->size(1)), static_cast<int32_t>(dim),
          static_cast<int32_t>(2 * cos->size(1)), args[8] == Py_True, cos->size(0), eps};
  return dim <= 1024;
}

PyObject* qk_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    NormCall c;
    if (n != 9 || !norm_call(args, dev, &c)) return nullptr;
    const at::Tensor q = dense_like(*c.q), k = dense_like(*c.k);
    c.a.q_out = heads_of(q), c.a.k_out = heads_of(k);
    return result_of(dev, [&](hipStream_t s) { return g_attention.norm(&c.a, s); }, [&] { return tuple_of({q, k}); });
  });
}

PyObject* qk_norm_rope_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    NormCall c;
    if (n != 11 || !norm_call(args + 2, dev, &c)) return nullptr;
    const at::Tensor *gq = on_device(args[0], dev), *gk = on_device(args[1], dev);
    if (!is_heads(gq) || !is_heads(gk) || gq->sizes() != c.q->sizes() || gk->sizes() != c.k->sizes()) return nullptr;
    c.a.q_out = heads_of(*gq), c.a.k_out = heads_of(*gk);
    const int64_t bytes = g_attention.norm_backward_workspace(&c.a);
    if (bytes < 0) return nullptr;
    const at::Tensor dq = dense_like(*c.q), dk = dense_like(*c.k), weights = at::empty({2, c.q->size(2)}, c.q->options().dtype(at::kFloat)), work = workspace(bytes, *c.q);
    const swz_heads hq = heads_of(dq), hk = heads_of(dk);
    float* w = static_cast<float*>(weights.data_ptr());
    return result_of(dev, [&](hipStream_t s) { return g_attention.norm_backward(&c.a, &hq, &hk, w, w + c.a.head_dim, work.data_ptr(), bytes, s); },
                     [&] { return tuple_of({dq, dk, weights.select(0, 0), weights.select(0, 1)}); });
  });
}

// args: q, k, v, cu_q, cu_k, causal, scale (None: the default)
struct PromptCall {
  const at::Tensor *q, *k, *v;
  swz_attention_args a;
};
bool prompt_call(PyObject* const* args, PyObject* const* flags, c10::DeviceIndex dev, PromptCall* c) {
  c->q = on_device(args[0], dev), c->k = on_device(args[1], dev), c->v = on_device(args[2], dev);
  const at::Tensor *cu_q = plain(flags[0], dev), *cu_k = flags[1] == Py_None ? cu_q : plain(flags[1], dev);
  if (!is_heads(c->q) || !is_heads(c->k) || !is_heads(c->v) || c->k->sizes() != c->v->sizes() || c->q->size(2) != c->k->size(2)) return false;
  if (!is_type(cu_q, 1, at::kInt) || cu_q->size(0) < 2 || cu_q->size(0) > (1 << 30) || !is_ints(cu_k, cu_q->size(0)) || !PyBool_Check(flags[2])) return false;
  const int64_t dim = c->q->size(2);
  if (dim > 1024 || c->q->size(1) > (1 << 20) || c->k->size(1) > (1 << 20)) return false;
  float scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(dim)));
  if (flags[3] != Py_None && !as_float(flags[3], &scale)) return false;
  c->a = {heads_of(*c->q), heads_of(*c->k), heads_of(*c->v), {}, nullptr, static_cast<const int32_t*>(cu_q->data_ptr()), static_cast<const int32_t*>(cu_k->data_ptr()),
          c->q->size(0), c->k->size(0), static_cast<int32_t>(cu_q->size(0) - 1), static_cast<int32_t>(c->q->size(1)), static_cast<int32_t>(c->k->size(1)),
          static_cast<int32_t>(dim), flags[2] == Py_True, scale};
  return true;
}

PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    PromptCall c;
    if (n != 7 || !prompt_call(args, args + 3, dev, &c)) return nullptr;
    const at::Tensor out = dense_like(*c.q), lse = at::empty({c.q->size(1), c.q->size(0)}, c.q->options().dtype(at::kFloat));
    c.a.out = heads_of(out), c.a.lse = static_cast<float*>(lse.data_ptr());
    const int64_t bytes = g_attention.attention_workspace(&c.a);
    if (bytes < 0) return nullptr;
    const at::Tensor work = bytes > 0 ? workspace(bytes, *c.q) : at::Tensor();
    return result_of(dev, [&](hipStream_t s) { return g_attention.attention(&c.a, bytes > 0 ? work.data_ptr() : nullptr, bytes, s); }, [&] { return tuple_of({out, lse}); });
  });
}

// args: dout, q, k, v, out, lse, cu_q, cu_k, causal, scale
PyObject* attention_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    PromptCall c;
    if (n != 10 || !prompt_call(args + 1, args + 6, dev, &c)) return nullptr;
    const at::Tensor *dout = on_device(args[0], dev), *out = on_device(args[4], dev), *lse = plain(args[5], dev);
    if (!is_heads(dout) || !is_heads(out) || dout->sizes() != c.q->sizes() || out->sizes() != c.q->sizes()) return nullptr;
    if (!is_type(lse, 2, at::kFloat) || lse->size(0) != c.q->size(1) || lse->size(1) != c.q->size(0)) return nullptr;
    c.a.out = heads_of(*out), c.a.lse = static_cast<float*>(lse->data_ptr());
    const int64_t bytes = g_attention.attention_backward_workspace(&c.a);
    if (bytes < 0) return nullptr;
    const at::Tensor dq = dense_like(*c.q), dk = dense_like(*c.k), dv = dense_like(*c.v), work = workspace(bytes, *c.q);
    const swz_heads g = heads_of(*dout), hq = heads_of(dq), hk = heads_of(dk), hv = heads_of(dv);
    return result_of(dev, [&](hipStream_t s) { return g_attention.attention_backward(&c.a, &g, &hq, &hk, &hv, work.data_ptr(), bytes, s); },
                     [&] { return tuple_of({dq, dk, dv}); });
  });
}

bool cache_of(PyObject* o, c10::DeviceIndex dev, swz_cache4* c) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i) t[i] = plain(PyTuple_GET_ITEM(o, i), dev);
  if (!is_type(t[0], 4, at::kInt) || !is_type(t[1], 4, at::kInt) || !is_type(t[2], 5, at::kBFloat16) || !is_type(t[3], 5, at::kBFloat16)) return false;
  const int64_t pages = t[0]->size(0), heads = t[0]->size(1), page = t[0]->size(2), dim = 8 * t[0]->size(3);
  if (page > (1 << 30) || heads > (1 << 20) || dim > 1024) return false;
  const int64_t v[4] = {pages, heads, page / 8, dim}, scales[5] = {pages, heads, page, dim / 64, 2};
  if (t[1]->sizes() != at::IntArrayRef(v, 4) || t[2]->sizes() != at::IntArrayRef(scales, 5) || t[3]->sizes() != t[2]->sizes()) return false;
  *c = {static_cast<int32_t*>(t[0]->data_ptr()), static_cast<int32_t*>(t[1]->data_ptr()), t[2]->data_ptr(), t[3]->data_ptr(), pages, static_cast<int32_t>(page),
        static_cast<int32_t>(heads), static_cast<int32_t>(dim)};
  return true;
}

// The sequences of a call on the cache: cu (or none), what each has, the table.
struct Sequences {
  const int32_t *cu, *counts, *table;
  int32_t n, width;
};
bool sequences_of(PyObject* cu_o, PyObject* counts_o, PyObject* table_o, c10::DeviceIndex dev, Sequences* s) {
  const at::Tensor *cu = cu_o == nullptr ? nullptr : plain(cu_o, dev), *counts = plain(counts_o, dev), *table = plain(table_o, dev);
  if (!is_type(counts, 1, at::kInt) || !is_type(table, 2, at::kInt) || table->size(0) != counts->size(0) || counts->size(0) < 1 || counts->size(0) > (1 << 30)) return false;
  if ((cu_o != nullptr && !is_ints(cu, counts->size(0) + 1)) || table->size(1) > (1 << 30)) return false;
  *s = {cu == nullptr ? nullptr : static_cast<const int32_t*>(cu->data_ptr()), static_cast<const int32_t*>(counts->data_ptr()), static_cast<const int32_t*>(table->data_ptr()),
        static_cast<int32_t>(counts->size(0)), static_cast<int32_t>(table->size(1))};
  return true;
}

// args: cache, k, v, cu, before, block_table; a status
PyObject* cache4_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    swz_cache4 c;
    Sequences s;
    if (n != 6 || !cache_of(args[0], dev, &c) || !sequences_of(args[3], args[4], args[5], dev, &s)) return nullptr;
    const at::Tensor *k = on_device(args[1], dev), *v = on_device(args[2], dev);
    if (!is_heads(k) || !is_heads(v) || k->sizes() != v->sizes() || k->size(1) != c.k_heads || k->size(2) != c.head_dim) return nullptr;
    const swz_heads hk = heads_of(*k), hv = heads_of(*v);
    const int64_t tokens = k->size(0);
    return launch(dev, [&](hipStream_t st) { return g_attention.append(&c, &hk, &hv, tokens, s.cu, s.counts, s.table, s.width, s.n, st); });
  });
}

// args: cache, cu, first, block_table, tokens
PyObject* cache4_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    swz_cache4 c;
    Sequences s;
    int tokens;
    if (n != 5 || !cache_of(args[0], dev, &c) || !sequences_of(args[1], args[2], args[3], dev, &s) || !as_int(args[4], &tokens) || tokens < 1) return nullptr;
    const at::TensorOptions options = THPVariable_Unpack(args[1]).options().dtype(at::kBFloat16);
    const at::Tensor k = at::empty({tokens, c.k_heads, c.head_dim}, options), v = at::empty({tokens, c.k_heads, c.head_dim}, options);
    const swz_heads hk = heads_of(k), hv = heads_of(v);
    return result_of(dev, [&](hipStream_t st) { return g_attention.read(&c, &hk, &hv, tokens, s.cu, s.counts, s.table, s.width, s.n, st); }, [&] { return tuple_of({k, v}); });
  });
}

// args: q, cache, lengths, block_table, max_length, scale
PyObject* cache4_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const c10::DeviceIndex dev = c10::hip::current_device();
    swz_cache4 c;
    Sequences s;
    int longest;
    if (n != 6 || !cache_of(args[1], dev, &c) || !sequences_of(nullptr, args[2], args[3], dev, &s) || !as_int(args[4], &longest)) return nullptr;
    const at::Tensor* q = on_device(args[0], dev);
    float scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(c.head_dim)));
    if (!is_heads(q) || q->size(0) != s.n || q->size(2) != c.head_dim || q->size(1) > (1 << 20) || (args[5] != Py_None && !as_float(args[5], &scale))) return nullptr;
    const int32_t heads = static_cast<int32_t>(q->size(1));
    const int64_t bytes = g_attention.cache_attention_workspace(&c, s.n, heads, s.width, longest);
    if (bytes < 0) return nullptr;
    const at::Tensor out = dense_like(*q), work = workspace(bytes, *q);
    const swz_heads hq = heads_of(*q), ho = heads_of(out);
    return result_of(dev, [&](hipStream_t st) { return g_attention.cache_attention(&c, &hq, &ho, s.counts, s.table, s.width, s.n, heads, longest, scale, work.data_ptr(), bytes, st); },
                     [&] { return THPVariable_Wrap(out); });
  });
}

// The library's functions, in the order of AttentionFns.
PyObject* bind_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr Py_ssize_t kCount = sizeof(AttentionFns) / sizeof(void*);
  void* p[kCount];
  if (n != kCount) {
    PyErr_SetString(PyExc_TypeError, "bind_attention takes one address for each function");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < kCount; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function");
      return nullptr;
    }
  }
  std::memcpy(&g_attention, p, sizeof p);
  Py_RETURN_NONE;
}

// The library's functions, as ctypes found them: this module links to no second copy of it.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* p[4];
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "bind(gemm, transpose, softmax, layernorm, Parameter)");
    return nullptr;
  }
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function");
      return nullptr;
    }
  }
  g_gemm = reinterpret_cast<GemmFn>(p[0]);
  g_transpose = reinterpret_cast<TransposeFn>(p[1]);
  g_softmax = reinterpret_cast<SoftmaxFn>(p[2]);
  g_layernorm = reinterpret_cast<LayernormFn>(p[3]);
  Py_INCREF(args[4]);
  Py_XSETREF(g_parameter, args[4]);
  Py_RETURN_NONE;
}

#define SWZ_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {SWZ_FAST(gemm), SWZ_FAST(transpose), SWZ_FAST(softmax), SWZ_FAST(layernorm), SWZ_FAST(bind),
                          SWZ_FAST(qk_norm_rope), SWZ_FAST(qk_norm_rope_backward), SWZ_FAST(attention), SWZ_FAST(attention_backward), SWZ_FAST(cache4_append),
                          SWZ_FAST(cache4_read), SWZ_FAST(cache4_attention), SWZ_FAST(bind_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() {
  PyObject* m = PyModule_Create(&kModule);
  if (m != nullptr && PyModule_AddStringConstant(m, "built_for", SWZ_TORCH_TAG) != 0) Py_CLEAR(m);       // binding.py uses it with that torch only
  return m;
}
