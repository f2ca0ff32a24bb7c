// Marshalling of the calls that a forward pass is made of, without the interpreter: tensor checks, sizes, the output's allocation
// and the call of the C entry point.  The Python functions in __init__.py are the reference for every check: a call that this file does
// not take as it is (another tensor class, a host tensor, strides, mixed types, sizes that do not fit) comes back as None and
// goes through them, so what is refused, and how, is written once.
//
// Per call, us (marshalling in Python -> here; of both 3.5 are the launch): linear 5.3 to 5.9 -> 3.8 with an output given, 7.5 -> 4.6 with one allocated; conv2d 8.2 -> 4.7.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>

#include "../../include/netfuse.h"

namespace {

decltype(&netfuse_linear) f_linear, f_packed;
decltype(&netfuse_layernorm) f_layernorm;
decltype(&netfuse_attention) f_attention;
decltype(&netfuse_attention_relpos) f_relpos;
decltype(&netfuse_conv2d) f_conv2d;
decltype(&netfuse_attention_prompt) f_prompt;
decltype(&netfuse_attention_tree) f_tree;
decltype(&netfuse_attention_tree_workspace) f_tree_workspace;
decltype(&netfuse_cache_append) f_append;
decltype(&netfuse_cache_weigh) f_weigh;
decltype(&netfuse_cache_evict) f_evict;
decltype(&netfuse_cache_evict_workspace) f_evict_workspace;
decltype(&netfuse_rotate_heads) f_rotate;
decltype(&netfuse_cache_append_fp4) f_append_fp4;
decltype(&netfuse_cache_read_fp4) f_read_fp4;
decltype(&netfuse_attention_tree_fp4) f_tree_fp4;
decltype(&netfuse_attention_tree_fp4_workspace) f_tree_fp4_workspace;
decltype(&netfuse_token_logprobs) f_logprobs;
decltype(&netfuse_token_logprobs_workspace) f_logprobs_workspace;
PyObject* g_error;                           // callable (entry point, status) that raises

const c10::DispatchKeySet kWrapped({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                    c10::DispatchKey::Functionalize});

// A tensor whose data pointer is what the kernels may read: cuda, contiguous, float32 or bfloat16, not a wrapper.
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.key_set().has_any(kWrapped) || !t.has_storage() || !t.is_contiguous()) return nullptr;
  const auto st = t.scalar_type();
  return st == at::kFloat || st == at::kBFloat16 ? &t : nullptr;
}
// An optional operand of type `st`: false if it is neither None nor that.
bool operand(PyObject* o, at::ScalarType st, void** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  if (!t || t->scalar_type() != st) return false;
  *p = t->data_ptr();
  return true;
}
bool whole(PyObject* o, int* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long x = PyLong_AsLongAndOverflow(o, &over);
  *v = (int)x;
  return !over && x == *v;
}
bool size(int64_t n, int* v) {
  *v = (int)n;
  return n == *v;
}
bool stream_of(PyObject* o, void** s) {
  if (!PyLong_CheckExact(o)) return false;
  *s = PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}
nf_dtype type_of(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? NF_F32 : NF_BF16; }

PyObject* not_taken() {
  PyErr_Clear();
  Py_RETURN_NONE;
}
PyObject* done(const char* fn, nf_status st, PyObject* given, at::Tensor& made) {
  if (st != NF_OK) {
    PyObject* r = PyObject_CallFunction(g_error, "si", fn, (int)st);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, fn);
    return nullptr;
  }
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(std::move(made));
}

// The interpreter's lock is not held while this lives.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  ~Unlocked() noexcept(false) { PyEval_RestoreThread(state); }   // a daemon thread may end here when the interpreter does
};
// The output and the call: call(y) on the tensor given, or on a new one.  The allocation may wait for memory and the launch for room
// in its queue, for as long as the work in front of it takes, so other Python threads run meanwhile, a host callback that the queue
// waits for among them (0.05 us).  `call` takes no Python object: every operand is a pointer by then.
template <class F>
PyObject* produce(const char* fn, PyObject* given, at::IntArrayRef shape, const at::TensorOptions& like, F&& call) {
  void* y = nullptr;
  if (!operand(given, at::typeMetaToScalarType(like.dtype()), &y)) return not_taken();
  at::Tensor made;
  nf_status st;
  {
    Unlocked unlocked;
    if (given == Py_None) {
      made = at::empty(shape, like);
      y = made.data_ptr();
    }
    st = call(y);
  }
  return done(fn, st, given, made);
}

// A C++ error (an allocation that fails) is met again, and raised as torch raises it, by the Python path.
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception&) {
    return not_taken();
  }
}

// X, W, bias, residual, act, out, stream
PyObject* matmul(decltype(f_linear) f, const char* name, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 7) return not_taken();
    const at::Tensor *X = plain(a[0]), *W = plain(a[1]);
    if (!X || !W || X->dim() != 3 || W->dim() != 3 || W->scalar_type() != X->scalar_type()) return not_taken();
    int M, N, K, No, act;
    void *b, *r, *s;
    if (!size(X->size(0), &M) || !size(X->size(1), &N) || !size(X->size(2), &K) || !size(W->size(2), &No) || W->size(0) != M ||
        W->size(1) != K || !operand(a[2], at::kFloat, &b) || !operand(a[3], X->scalar_type(), &r) || !whole(a[4], &act) || !stream_of(a[6], &s))
      return not_taken();
    const void *x = X->data_ptr(), *w = W->data_ptr();
    const nf_dtype dt = type_of(*X);
    return produce(name, a[5], {M, N, No}, X->options(), [=](void* y) { return f(x, w, (const float*)b, r, y, M, N, K, No, dt, (nf_act)act, s); });
  });
}
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) { return matmul(f_linear, "netfuse_linear", a, n); }
PyObject* linear_packed(PyObject*, PyObject* const* a, Py_ssize_t n) { return matmul(f_packed, "netfuse_linear_packed", a, n); }

// x, gamma, beta, M, residual, eps, layout, out, stream
PyObject* layernorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9) return not_taken();
    const at::Tensor* x = plain(a[0]);
    int M, layout, rows, H;
    void *g, *b, *r, *s;
    if (!x || !whole(a[3], &M) || M <= 0 || !whole(a[6], &layout) || !PyFloat_CheckExact(a[5]) || !operand(a[1], at::kFloat, &g) ||
        !operand(a[2], at::kFloat, &b) || !operand(a[4], x->scalar_type(), &r) || !stream_of(a[8], &s))
      return not_taken();
    if (layout == NF_MERGE_BATCH) {
      if (x->dim() != 3 || !size(x->size(1), &rows) || !size(x->size(2), &H)) return not_taken();
    } else if (x->dim() != 2 || !size(x->size(0), &rows) || !size(x->size(1) / M, &H)) {
      return not_taken();
    }
    const void* in = x->data_ptr();
    const float eps = (float)PyFloat_AS_DOUBLE(a[5]);
    const nf_dtype dt = type_of(*x);
    const at::DimVector shape(x->sizes());
    return produce("netfuse_layernorm", a[7], shape, x->options(), [=](void* y) {
      return f_layernorm(in, r, (const float*)g, (const float*)b, y, M, rows, H, eps, (nf_merge_dim)layout, dt, s);
    });
  });
}

// QKV[M][B*S][3 heads d] with its scale: the shape checks of both attentions
bool packed_qkv(const at::Tensor& t, PyObject* B_, PyObject* S_, PyObject* heads_, PyObject* scale_, int* M, int* B, int* S, int* heads, int* d,
                float* scale) {
  int N, H3;
  if (t.dim() != 3 || !whole(B_, B) || !whole(S_, S) || !whole(heads_, heads) || *heads <= 0 || !size(t.size(0), M) || !size(t.size(1), &N) ||
      !size(t.size(2), &H3))
    return false;
  *d = H3 / 3 / *heads;
  if (N != (int64_t)*B * *S || H3 != 3LL * *heads * *d || *d <= 0) return false;
  if (scale_ == Py_None) *scale = (float)std::pow((double)*d, -0.5);
  else if (PyFloat_CheckExact(scale_)) *scale = (float)PyFloat_AS_DOUBLE(scale_);
  else return false;
  return true;
}
// QKV, B, S, heads, scale, mask, out, stream
PyObject* attention_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 8) return not_taken();
    const at::Tensor* Q = plain(a[0]);
    int M, B, S, heads, d;
    float scale;
    void *mask, *s;
    if (!Q || !packed_qkv(*Q, a[1], a[2], a[3], a[4], &M, &B, &S, &heads, &d, &scale) || !operand(a[5], at::kFloat, &mask) || !stream_of(a[7], &s))
      return not_taken();
    const long Hd = (long)heads * d, N = (long)B * S;
    const char* base = (const char*)Q->data_ptr();
    const long step = Hd * (long)Q->element_size();
    const nf_dtype dt = type_of(*Q);
    return produce("netfuse_attention", a[6], {M, N, Hd}, Q->options(), [=](void* y) {
      return f_attention(base, base + step, base + 2 * step, (const float*)mask, y, M, B, S, heads, d, N * 3 * Hd, 3 * Hd, scale, dt, s);
    });
  });
}
// QKV, Kr, B, S, heads, bias_w, bias_r, scale, mask, out, stream
PyObject* attention_relpos_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 11) return not_taken();
    const at::Tensor *Q = plain(a[0]), *Kr = plain(a[1]);
    int M, B, S, heads, d;
    float scale;
    void *bw, *br, *mask, *s;
    if (!Q || !Kr || Kr->scalar_type() != Q->scalar_type() || !packed_qkv(*Q, a[2], a[3], a[4], a[7], &M, &B, &S, &heads, &d, &scale) ||
        !operand(a[5], at::kFloat, &bw) || !operand(a[6], at::kFloat, &br) || !operand(a[8], at::kFloat, &mask) || !stream_of(a[10], &s))
      return not_taken();
    const long Hd = (long)heads * d, N = (long)B * S;
    if (Kr->dim() != 3 || Kr->size(0) != M || Kr->size(1) != 2LL * S || Kr->size(2) != Hd) return not_taken();
    const char* base = (const char*)Q->data_ptr();
    const void* kr = Kr->data_ptr();
    const long step = Hd * (long)Q->element_size();
    const nf_dtype dt = type_of(*Q);
    return produce("netfuse_attention_relpos", a[9], {M, N, Hd}, Q->options(), [=](void* y) {
      return f_relpos(base, base + step, base + 2 * step, kr, (const float*)bw, (const float*)br, (const float*)mask, y, M, B, S, heads, d,
                      N * 3 * Hd, 3 * Hd, scale, dt, s);
    });
  });
}

// x, w, M, g, bias, scale, shift, residual, stride, pad, dil, act, out, stream
PyObject* conv2d(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 14) return not_taken();
    const at::Tensor *x = plain(a[0]), *w = plain(a[1]);
    int M, g, stride, pad, dil, act, B, Ct, H, W, Co, cig, KH, KW;
    void *bias, *scale, *shift, *r, *s;
    if (!x || !w || x->dim() != 4 || w->dim() != 4 || w->scalar_type() != x->scalar_type() || !whole(a[2], &M) || M <= 0 || !whole(a[3], &g) || g <= 0 ||
        !operand(a[4], at::kFloat, &bias) || !operand(a[5], at::kFloat, &scale) || !operand(a[6], at::kFloat, &shift) ||
        !operand(a[7], x->scalar_type(), &r) || !whole(a[8], &stride) || stride <= 0 || !whole(a[9], &pad) || pad < 0 || !whole(a[10], &dil) || dil <= 0 ||
        !whole(a[11], &act) || !stream_of(a[13], &s))
      return not_taken();
    if (!size(x->size(0), &B) || !size(x->size(1), &Ct) || !size(x->size(2), &H) || !size(x->size(3), &W) || !size(w->size(0), &Co) ||
        !size(w->size(1), &cig) || !size(w->size(2), &KH) || !size(w->size(3), &KW) || Ct % M || Co % M || (int64_t)cig * g != Ct / M)
      return not_taken();
    const int64_t eh = (int64_t)H + 2LL * pad - (int64_t)dil * (KH - 1) - 1, ew = (int64_t)W + 2LL * pad - (int64_t)dil * (KW - 1) - 1;
    if (eh < 0 || ew < 0) return not_taken();
    const void *in = x->data_ptr(), *wt = w->data_ptr();
    const nf_dtype dt = type_of(*x);
    return produce("netfuse_conv2d", a[12], {B, Co, eh / stride + 1, ew / stride + 1}, x->options(), [=](void* y) {
      return f_conv2d(in, wt, (const float*)bias, (const float*)scale, (const float*)shift, r, y, M, B, Ct / M, Co / M, g, H, W, KH, KW, stride, pad,
                      dil, dt, (nf_act)act, s);
    });
  });
}

// ---- decoders: every operand's shape, type and device is checked here, and what is not as it should be goes to decoder.py for its error

const at::Tensor* strided(PyObject* o, at::ScalarType st, int device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.key_set().has_any(kWrapped) || !t.has_storage() || t.scalar_type() != st ||
      t.device().index() != device)
    return nullptr;
  return &t;
}
// A contiguous operand of this type and shape, or None where it may be missing.
bool dense(PyObject* o, at::ScalarType st, at::IntArrayRef shape, int device, bool needed, void** p) {
  *p = nullptr;
  if (o == Py_None) return !needed;
  const at::Tensor* t = strided(o, st, device);
  if (!t || t->sizes() != shape || !t->is_contiguous()) return false;
  *p = t->data_ptr();
  return true;
}
struct Rows {
  const void* p;
  long model, row;
};
// [M][N][width] with a contiguous last dimension; the stride of a dimension of one element says nothing.
bool rows(const at::Tensor* t, int64_t M, int64_t N, int64_t width, Rows* r) {
  if (!t || t->dim() != 3 || t->size(0) != M || t->size(1) != N || t->size(2) != width || (width > 1 && t->stride(2) != 1)) return false;
  r->p = t->data_ptr();
  r->row = N > 1 ? t->stride(1) : width;
  r->model = M > 1 ? t->stride(0) : (N - 1) * r->row + width;
  return true;
}
bool number(PyObject* o, float* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = (float)PyFloat_AS_DOUBLE(o);
  return true;
}
bool scale_of(PyObject* o, int d, float* v) {
  if (o == Py_None) {
    *v = (float)std::pow((double)d, -0.5);
    return true;
  }
  return number(o, v);
}
// The type of the rows and the current device.
bool types(PyObject* o, PyObject* device_, at::ScalarType* st, int* device) {
  if (!THPVariable_CheckExact(o) || !whole(device_, device)) return false;
  *st = THPVariable_Unpack(o).scalar_type();
  return *st == at::kFloat || *st == at::kBFloat16;
}
struct Cache {
  int M, B, kv, C, d;
  void* p;
};
bool cache(PyObject* o, at::ScalarType st, int device, Cache* c) {
  const at::Tensor* t = strided(o, st, device);
  if (!t || t->dim() != 5 || !t->is_contiguous() || !size(t->size(0), &c->M) || !size(t->size(1), &c->B) || !size(t->size(2), &c->kv) || !size(t->size(3), &c->C) ||
      !size(t->size(4), &c->d) || t->numel() == 0)
    return false;
  c->p = t->data_ptr();
  return true;
}
// Rows of a batch of c.B sequences: T of them each.
bool batch(const at::Tensor* t, const Cache& c, int* T) { return t && t->dim() == 3 && t->size(1) > 0 && t->size(1) % c.B == 0 && size(t->size(1) / c.B, T); }

// Q, K, V, B, S, heads, kv_heads, causal, scale, cap, slope, length, prefix, doc, out, device, stream
PyObject* attention_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, B, S, heads, kv, M, d;
    float scale, cap;
    void *slope, *len, *prefix, *doc, *s;
    if (n != 17 || !types(a[0], a[15], &st, &device)) return not_taken();
    const at::Tensor *Q = strided(a[0], st, device), *K = strided(a[1], st, device), *V = strided(a[2], st, device);
    if (!Q || Q->dim() != 3 || !whole(a[3], &B) || !whole(a[4], &S) || !whole(a[5], &heads) || B <= 0 || S <= 0 || heads <= 0 || !size(Q->size(0), &M) || M <= 0 ||
        Q->size(2) % heads || !size(Q->size(2) / heads, &d) || d <= 0 || !PyBool_Check(a[7]) || !scale_of(a[8], d, &scale) || !number(a[9], &cap) || !stream_of(a[16], &s))
      return not_taken();
    kv = heads;
    if (a[6] != Py_None && (!whole(a[6], &kv) || kv <= 0)) return not_taken();
    Rows q, k, v;
    const int64_t N = (int64_t)B * S;
    if (!rows(Q, M, N, (int64_t)heads * d, &q) || !rows(K, M, N, (int64_t)kv * d, &k) || !rows(V, M, N, (int64_t)kv * d, &v) || k.model != v.model || k.row != v.row ||
        !dense(a[10], at::kFloat, {M, heads}, device, false, &slope) || !dense(a[11], at::kInt, {M, B}, device, false, &len) ||
        !dense(a[12], at::kInt, {M, B}, device, false, &prefix) || !dense(a[13], at::kInt, {M, B, S}, device, false, &doc))
      return not_taken();
    void* given;
    if (!dense(a[14], st, {M, N, (int64_t)heads * d}, device, false, &given)) return not_taken();
    const int causal = a[7] == Py_True;
    const nf_dtype dt = type_of(*Q);
    return produce("netfuse_attention_prompt", a[14], {M, N, (int64_t)heads * d}, Q->options(), [=](void* y) {
      return f_prompt(q.p, k.p, v.p, (const float*)slope, (const int*)len, (const int*)prefix, (const int*)doc, y, M, B, S, heads, kv, d, q.model, q.row, k.model, k.row, causal, scale, cap,
                      dt, s);
    });
  });
}

// Q, K, V, Kc, Vc, length, start, parent, nodes, pos, slope, scale, cap, out, lse, workspace, device, stream
PyObject* attention_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, T, heads;
    float scale, cap;
    void *vc, *len, *start, *parent, *nodes, *pos, *slope, *given, *lse, *ws = nullptr, *s;
    Cache c;
    if (n != 18 || !types(a[0], a[16], &st, &device) || !cache(a[3], st, device, &c) || !dense(a[4], st, {c.M, c.B, c.kv, c.C, c.d}, device, true, &vc)) return not_taken();
    const at::Tensor *Q = strided(a[0], st, device), *K = strided(a[1], st, device), *V = strided(a[2], st, device);
    if (!batch(Q, c, &T) || Q->size(2) % c.d || !size(Q->size(2) / c.d, &heads) || !scale_of(a[11], c.d, &scale) || !number(a[12], &cap) || !stream_of(a[17], &s)) return not_taken();
    Rows q, k, v;
    const int64_t N = (int64_t)c.B * T, W = (int64_t)heads * c.d;
    if (!rows(Q, c.M, N, W, &q) || !rows(K, c.M, N, (int64_t)c.kv * c.d, &k) || !rows(V, c.M, N, (int64_t)c.kv * c.d, &v) || k.model != v.model || k.row != v.row ||
        !dense(a[5], at::kInt, {c.M, c.B}, device, true, &len) || !dense(a[6], at::kInt, {c.M, c.B}, device, false, &start) ||
        !dense(a[7], at::kInt, {c.M, c.B, T}, device, false, &parent) || !dense(a[8], at::kInt, {c.M, c.B}, device, false, &nodes) ||
        !dense(a[9], at::kInt, {c.M, c.B, c.kv, c.C}, device, false, &pos) || !dense(a[10], at::kFloat, {c.M, heads}, device, false, &slope) ||
        !dense(a[13], st, {c.M, N, W}, device, false, &given) || !dense(a[14], at::kFloat, {c.M, N, heads}, device, false, &lse))
      return not_taken();
    const nf_dtype dt = type_of(*Q);
    long long bytes = f_tree_workspace(c.M, c.B, T, c.C, heads, c.kv, c.d, dt);
    if (bytes < 0) return not_taken();
    at::Tensor room;
    const bool mine = a[15] == Py_None && bytes > 0;
    if (a[15] != Py_None) {
      if (!THPVariable_CheckExact(a[15])) return not_taken();
      const at::Tensor& w = THPVariable_Unpack(a[15]);
      if (!w.defined() || !w.is_cuda() || w.layout() != at::kStrided || w.key_set().has_any(kWrapped) || !w.has_storage() || !w.is_contiguous() || w.device().index() != device) return not_taken();
      ws = w.data_ptr();
      bytes = w.numel() * (long long)w.element_size();
    }
    return produce("netfuse_attention_tree", a[13], {c.M, N, W}, Q->options(), [&](void* y) {
      if (mine) {
        room = at::empty({bytes}, Q->options().dtype(at::kByte));
        ws = room.data_ptr();
      }
      return f_tree(q.p, k.p, v.p, c.p, vc, (const int*)pos, (const int*)len, (const int*)start, (const int*)parent, (const int*)nodes, (const float*)slope, y, (float*)lse, ws, bytes, c.M, c.B, T,
                    c.C, heads, c.kv, c.d, q.model, q.row, k.model, k.row, scale, cap, dt, s);
    });
  });
}

// A call that has no output of its own: True where it was made.
template <class F>
PyObject* made(const char* fn, F&& call) {
  nf_status st;
  {
    Unlocked unlocked;
    st = call();
  }
  at::Tensor none;
  return done(fn, st, Py_True, none);
}

// K, V, Kc, Vc, pos, weight, length, start, index, count, device, stream
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, T, m;
    void *vc, *pos, *weight, *len, *start, *index, *count, *s;
    Cache c;
    if (n != 12 || !types(a[0], a[10], &st, &device) || !cache(a[2], st, device, &c) || !dense(a[3], st, {c.M, c.B, c.kv, c.C, c.d}, device, true, &vc) || !stream_of(a[11], &s)) return not_taken();
    const at::Tensor *K = strided(a[0], st, device), *V = strided(a[1], st, device);
    if (!batch(K, c, &T)) return not_taken();
    m = T;
    if (a[8] != Py_None) {
      const at::Tensor* i = strided(a[8], at::kInt, device);
      if (!i || i->dim() != 3 || !size(i->size(2), &m)) return not_taken();
    }
    Rows k, v;
    const int64_t N = (int64_t)c.B * T, W = (int64_t)c.kv * c.d;
    if (!rows(K, c.M, N, W, &k) || !rows(V, c.M, N, W, &v) || k.model != v.model || k.row != v.row || !dense(a[4], at::kInt, {c.M, c.B, c.kv, c.C}, device, false, &pos) ||
        !dense(a[5], at::kFloat, {c.M, c.B, c.kv, c.C}, device, false, &weight) || !dense(a[6], at::kInt, {c.M, c.B}, device, true, &len) ||
        !dense(a[7], at::kInt, {c.M, c.B}, device, false, &start) || !dense(a[8], at::kInt, {c.M, c.B, m}, device, false, &index) ||
        !dense(a[9], at::kInt, {c.M, c.B}, device, false, &count))
      return not_taken();
    const nf_dtype dt = type_of(*K);
    return made("netfuse_cache_append", [=] {
      return f_append(k.p, v.p, (const int*)index, (const int*)count, (const int*)len, (const int*)start, c.p, vc, (int*)pos, (float*)weight, c.M, c.B, T, m, c.C, c.kv, c.d, k.model, k.row, dt, s);
    });
  });
}

// Q, lse, Kc, weight, length, start, index, count, pos, slope, scale, cap, out, device, stream
PyObject* cache_weigh(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, T, m, heads;
    float scale, cap;
    void *lse, *weight, *len, *start, *index, *count, *pos, *slope, *given, *s;
    Cache c;
    if (n != 15 || !types(a[0], a[13], &st, &device) || !cache(a[2], st, device, &c) || !stream_of(a[14], &s)) return not_taken();
    const at::Tensor* Q = strided(a[0], st, device);
    if (!batch(Q, c, &T) || Q->size(2) % c.d || !size(Q->size(2) / c.d, &heads) || !scale_of(a[10], c.d, &scale) || !number(a[11], &cap)) return not_taken();
    m = T;
    if (a[6] != Py_None) {
      const at::Tensor* i = strided(a[6], at::kInt, device);
      if (!i || i->dim() != 3 || !size(i->size(2), &m)) return not_taken();
    }
    Rows q;
    const int64_t N = (int64_t)c.B * T;
    const at::DimVector shape({c.M, c.B, c.kv, c.C});
    if (!rows(Q, c.M, N, (int64_t)heads * c.d, &q) || !dense(a[1], at::kFloat, {c.M, N, heads}, device, true, &lse) || !dense(a[3], at::kFloat, shape, device, true, &weight) ||
        !dense(a[4], at::kInt, {c.M, c.B}, device, true, &len) || !dense(a[5], at::kInt, {c.M, c.B}, device, false, &start) ||
        !dense(a[6], at::kInt, {c.M, c.B, m}, device, false, &index) || !dense(a[7], at::kInt, {c.M, c.B}, device, false, &count) || !dense(a[8], at::kInt, shape, device, false, &pos) ||
        !dense(a[9], at::kFloat, {c.M, heads}, device, false, &slope) || !dense(a[12], at::kFloat, shape, device, false, &given))
      return not_taken();
    const nf_dtype dt = type_of(*Q);
    return produce("netfuse_cache_weigh", a[12], shape, Q->options().dtype(at::kFloat), [=](void* y) {
      return f_weigh(q.p, (const float*)lse, (const int*)index, (const int*)count, c.p, (const int*)pos, (const int*)len, (const int*)start, (const float*)slope, (const float*)weight, (float*)y, c.M, c.B,
                     T, m, c.C, heads, c.kv, c.d, q.model, q.row, scale, cap, dt, s);
    });
  });
}

// Kc, Vc, pos, weight, length, budget, start, recent, pos_out, weight_out, device, stream (a workspace of the caller's is decoder.py's)
PyObject* cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, budget, recent;
    void *vc, *pos, *weight, *len, *start, *pos_out, *weight_out, *s;
    Cache c;
    if (n != 12 || !types(a[0], a[10], &st, &device) || !cache(a[0], st, device, &c) || !dense(a[1], st, {c.M, c.B, c.kv, c.C, c.d}, device, true, &vc) || !whole(a[5], &budget) ||
        !whole(a[7], &recent) || !stream_of(a[11], &s))
      return not_taken();
    const at::DimVector shape({c.M, c.B, c.kv, c.C});
    if (!dense(a[2], at::kInt, shape, device, false, &pos) || !dense(a[3], at::kFloat, shape, device, true, &weight) || !dense(a[4], at::kInt, {c.M, c.B}, device, true, &len) ||
        !dense(a[6], at::kInt, {c.M, c.B}, device, false, &start) || !dense(a[8], at::kInt, shape, device, false, &pos_out) || !dense(a[9], at::kFloat, shape, device, true, &weight_out))
      return not_taken();
    const at::Tensor& K = THPVariable_Unpack(a[0]);
    const nf_dtype dt = type_of(K);
    const long long bytes = f_evict_workspace(c.M, c.B, c.C, c.kv, budget);
    if (bytes < 0) return not_taken();
    at::Tensor room;
    return made("netfuse_cache_evict", [&] {
      room = at::empty({bytes}, K.options().dtype(at::kByte));
      return f_evict(c.p, vc, (const int*)pos, (const float*)weight, (const int*)len, (const int*)start, (int*)pos_out, (float*)weight_out, room.data_ptr(), bytes, c.M, c.B, c.C, c.kv, c.d, budget,
                     recent, dt, s);
    });
  });
}

// ---- a decoder's step around its attention: step.py, as above

// The caller's workspace, if any: its address, and its size in place of `bytes`.
bool workspace(PyObject* o, int device, void** p, long long* bytes) {
  *p = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& w = THPVariable_Unpack(o);
  if (!w.defined() || !w.is_cuda() || w.layout() != at::kStrided || w.key_set().has_any(kWrapped) || !w.has_storage() || !w.is_contiguous() || w.device().index() != device) return false;
  *p = w.data_ptr();
  *bytes = w.numel() * (long long)w.element_size();
  return true;
}
struct CacheFp4 {
  int M, B, kv, C, d;
  void *Kc, *Ks, *Vc, *Vs;
};
// Codes and scales of keys and, where `o` has them, of values, for heads of c->d features
bool cache_fp4(PyObject* const* o, int device, bool values, CacheFp4* c) {
  const at::Tensor* t = strided(o[0], at::kByte, device);
  if (!t || t->dim() != 5 || !size(t->size(0), &c->M) || !size(t->size(1), &c->B) || !size(t->size(2), &c->kv) || !size(t->size(3), &c->C) || t->numel() == 0) return false;
  const int64_t G = (c->d + 31) / 32, codes = 16 * G, scales = G + G % 2;
  return dense(o[0], at::kByte, {c->M, c->B, c->kv, c->C, codes}, device, true, &c->Kc) && dense(o[1], at::kByte, {c->M, c->B, c->kv, c->C, scales}, device, true, &c->Ks) &&
         dense(o[2], at::kByte, {c->M, c->B, c->kv, c->C, codes}, device, values, &c->Vc) && dense(o[3], at::kByte, {c->M, c->B, c->kv, c->C, scales}, device, values, &c->Vs);
}
// Features of a head: of rows of kv heads, kv the third size of the codes
bool head_size(const at::Tensor* rows, PyObject* codes, int device, int* d) {
  const at::Tensor* t = strided(codes, at::kByte, device);
  return rows && rows->dim() == 3 && t && t->dim() == 5 && t->size(2) > 0 && rows->size(2) > 0 && rows->size(2) % t->size(2) == 0 && size(rows->size(2) / t->size(2), d);
}

// Q, K, B, S, heads, kv_heads, freq, gamma_q, gamma_k, pos, start, length, sections, interleaved, eps, out_q, out_k, device, stream
PyObject* rotate_heads(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, B, S, heads, kv, M, d, pairs = 0, axes = 1, parts[4];
    float eps;
    void *gq, *gk, *freq, *pos, *start, *len, *s;
    if (n != 19 || !types(a[0], a[17], &st, &device)) return not_taken();
    const at::Tensor *Q = strided(a[0], st, device), *K = a[1] == Py_None ? nullptr : strided(a[1], st, device);
    if (!Q || (a[1] != Py_None && !K) || Q->dim() != 3 || !whole(a[2], &B) || !whole(a[3], &S) || !whole(a[4], &heads) || B <= 0 || S <= 0 || heads <= 0 || !size(Q->size(0), &M) || M <= 0 ||
        Q->size(2) % heads || !size(Q->size(2) / heads, &d) || d <= 0 || !PyBool_Check(a[13]) || !number(a[14], &eps) || !stream_of(a[18], &s))
      return not_taken();
    kv = heads;
    if (a[5] != Py_None && !whole(a[5], &kv)) return not_taken();
    if (!K) kv = 0;
    if (K && kv <= 0) return not_taken();
    if (a[6] != Py_None) {
      const at::Tensor* f = strided(a[6], at::kFloat, device);
      if (!f || f->dim() != 1 || !size(f->size(0), &pairs) || pairs > (1 << 20)) return not_taken();
    }
    if (a[12] != Py_None) {
      if (!PyList_CheckExact(a[12])) return not_taken();
      const Py_ssize_t count = PyList_GET_SIZE(a[12]);
      if (count < 1 || count > 4) return not_taken();
      axes = (int)count;
      for (int x = 0; x < axes; ++x)
        if (!whole(PyList_GET_ITEM(a[12], x), &parts[x])) return not_taken();
    }
    const int64_t N = (int64_t)B * S;
    if (a[9] == Py_None) {
      if (axes > 1) return not_taken();
      pos = nullptr;
    } else if (!dense(a[9], at::kInt, {M, B, S, axes}, device, true, &pos) && (axes > 1 || !dense(a[9], at::kInt, {M, B, S}, device, true, &pos))) {
      return not_taken();
    }
    Rows q, k = {nullptr, 0, 0}, qo, ko = {nullptr, 0, 0};
    if (!rows(Q, M, N, (int64_t)heads * d, &q) || (K && !rows(K, M, N, (int64_t)kv * d, &k)) || !dense(a[6], at::kFloat, {pairs}, device, false, &freq) ||
        !dense(a[7], at::kFloat, {M, d}, device, false, &gq) || !dense(a[8], at::kFloat, {M, d}, device, false, &gk) || !dense(a[10], at::kInt, {M, B}, device, false, &start) ||
        !dense(a[11], at::kInt, {M, B}, device, false, &len))
      return not_taken();
    // new results where no row of them is left out; with lengths step.py clears them
    at::Tensor new_q, new_k;
    const at::Tensor *Qo = nullptr, *Ko = nullptr;
    if (a[15] != Py_None ? !(Qo = strided(a[15], st, device)) : len != nullptr) return not_taken();
    if (K ? (a[16] != Py_None ? !(Ko = strided(a[16], st, device)) : len != nullptr) : a[16] != Py_None) return not_taken();
    if ((Qo && !rows(Qo, M, N, (int64_t)heads * d, &qo)) || (Ko && !rows(Ko, M, N, (int64_t)kv * d, &ko))) return not_taken();
    const int interleaved = a[13] == Py_True;
    const nf_dtype dt = type_of(*Q);
    nf_status done_as;
    {
      Unlocked unlocked;
      if (!Qo) {
        new_q = at::empty({M, N, (int64_t)heads * d}, Q->options());
        qo = {new_q.data_ptr(), (long)(N * heads * d), (long)heads * d};
      }
      if (K && !Ko) {
        new_k = at::empty({M, N, (int64_t)kv * d}, Q->options());
        ko = {new_k.data_ptr(), (long)(N * kv * d), (long)kv * d};
      }
      done_as = f_rotate(q.p, k.p, (const float*)gq, (const float*)gk, (const float*)freq, (const int*)pos, (const int*)start, (const int*)len, a[12] != Py_None ? parts : nullptr, (void*)qo.p,
                         (void*)ko.p, M, B, S, heads, kv, d, 2 * pairs, axes, q.model, q.row, k.model, k.row, qo.model, qo.row, ko.model, ko.row, eps, interleaved, dt, s);
    }
    PyObject* first = done("netfuse_rotate_heads", done_as, a[15], new_q);
    if (!first) return nullptr;
    PyObject* second = a[16];
    if (K && !Ko) second = THPVariable_Wrap(std::move(new_k));
    else Py_INCREF(second);
    PyObject* both = second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_DECREF(first);
    Py_XDECREF(second);
    return both;
  });
}

// K, V, Kc, Ks, Vc, Vs, pos, weight, length, start, index, count, device, stream
PyObject* cache_append_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, T, m;
    void *pos, *weight, *len, *start, *index, *count, *s;
    CacheFp4 c;
    if (n != 14 || !types(a[0], a[12], &st, &device) || !stream_of(a[13], &s)) return not_taken();
    const at::Tensor *K = strided(a[0], st, device), *V = strided(a[1], st, device);
    if (!head_size(K, a[2], device, &c.d) || !cache_fp4(a + 2, device, true, &c) || !batch(K, {c.M, c.B, c.kv, c.C, c.d, nullptr}, &T)) return not_taken();
    m = T;
    if (a[10] != Py_None) {
      const at::Tensor* i = strided(a[10], at::kInt, device);
      if (!i || i->dim() != 3 || !size(i->size(2), &m)) return not_taken();
    }
    Rows k, v;
    const int64_t N = (int64_t)c.B * T, W = (int64_t)c.kv * c.d;
    const at::DimVector shape({c.M, c.B, c.kv, c.C});
    if (!rows(K, c.M, N, W, &k) || !rows(V, c.M, N, W, &v) || k.model != v.model || k.row != v.row || !dense(a[6], at::kInt, shape, device, false, &pos) ||
        !dense(a[7], at::kFloat, shape, device, false, &weight) || !dense(a[8], at::kInt, {c.M, c.B}, device, true, &len) || !dense(a[9], at::kInt, {c.M, c.B}, device, false, &start) ||
        !dense(a[10], at::kInt, {c.M, c.B, m}, device, false, &index) || !dense(a[11], at::kInt, {c.M, c.B}, device, false, &count))
      return not_taken();
    const nf_dtype dt = type_of(*K);
    return made("netfuse_cache_append_fp4", [=] {
      return f_append_fp4(k.p, v.p, (const int*)index, (const int*)count, (const int*)len, (const int*)start, c.Kc, c.Ks, c.Vc, c.Vs, (int*)pos, (float*)weight, c.M, c.B, T, m, c.C, c.kv, c.d, k.model,
                          k.row, dt, s);
    });
  });
}

// Kc, Ks, Vc, Vs, d, n, first, count, out_k, out_v, device, stream (new results are step.py's)
PyObject* cache_read_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, m;
    void *first, *count, *k, *v, *s;
    CacheFp4 c;
    if (n != 12 || !types(a[8], a[10], &st, &device) || !stream_of(a[11], &s) || !whole(a[4], &c.d) || c.d <= 0 || c.d > 256) return not_taken();
    const bool values = a[9] != Py_None;
    if (!cache_fp4(a, device, values, &c) || (c.Vc != nullptr) != values || (c.Vs != nullptr) != values) return not_taken();
    m = c.C;
    if (a[5] != Py_None && (!whole(a[5], &m) || m <= 0)) return not_taken();
    const at::DimVector shape({c.M, c.B, c.kv, m, c.d});
    if (!dense(a[6], at::kInt, {c.M, c.B}, device, false, &first) || !dense(a[7], at::kInt, {c.M, c.B}, device, false, &count) || !dense(a[8], st, shape, device, true, &k) ||
        !dense(a[9], st, shape, device, false, &v))
      return not_taken();
    const nf_dtype dt = st == at::kFloat ? NF_F32 : NF_BF16;
    return made("netfuse_cache_read_fp4",
                [=] { return f_read_fp4(c.Kc, c.Ks, c.Vc, c.Vs, (const int*)first, (const int*)count, k, v, c.M, c.B, m, c.C, c.kv, c.d, dt, s); });
  });
}

// Q, K, V, Kc, Ks, Vc, Vs, length, start, parent, nodes, pos, slope, scale, cap, out, lse, workspace, device, stream
PyObject* attention_tree_fp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, T, heads;
    float scale, cap;
    void *len, *start, *parent, *nodes, *pos, *slope, *given, *lse, *ws, *s;
    CacheFp4 c;
    if (n != 20 || !types(a[0], a[18], &st, &device)) return not_taken();
    const at::Tensor *Q = strided(a[0], st, device), *K = strided(a[1], st, device), *V = strided(a[2], st, device);
    if (!head_size(K, a[3], device, &c.d) || !cache_fp4(a + 3, device, true, &c) || !batch(Q, {c.M, c.B, c.kv, c.C, c.d, nullptr}, &T) || Q->size(2) % c.d || !size(Q->size(2) / c.d, &heads) ||
        !scale_of(a[13], c.d, &scale) || !number(a[14], &cap) || !stream_of(a[19], &s))
      return not_taken();
    Rows q, k, v;
    const int64_t N = (int64_t)c.B * T, W = (int64_t)heads * c.d;
    if (!rows(Q, c.M, N, W, &q) || !rows(K, c.M, N, (int64_t)c.kv * c.d, &k) || !rows(V, c.M, N, (int64_t)c.kv * c.d, &v) || k.model != v.model || k.row != v.row ||
        !dense(a[7], at::kInt, {c.M, c.B}, device, true, &len) || !dense(a[8], at::kInt, {c.M, c.B}, device, false, &start) || !dense(a[9], at::kInt, {c.M, c.B, T}, device, false, &parent) ||
        !dense(a[10], at::kInt, {c.M, c.B}, device, false, &nodes) || !dense(a[11], at::kInt, {c.M, c.B, c.kv, c.C}, device, false, &pos) ||
        !dense(a[12], at::kFloat, {c.M, heads}, device, false, &slope) || !dense(a[15], st, {c.M, N, W}, device, false, &given) ||
        !dense(a[16], at::kFloat, {c.M, N, heads}, device, false, &lse))
      return not_taken();
    const nf_dtype dt = type_of(*Q);
    long long bytes = f_tree_fp4_workspace(c.M, c.B, T, c.C, heads, c.kv, c.d, dt);
    if (bytes < 0 || !workspace(a[17], device, &ws, &bytes)) return not_taken();
    at::Tensor room;
    const bool mine = a[17] == Py_None && bytes > 0;
    return produce("netfuse_attention_tree_fp4", a[15], {c.M, N, W}, Q->options(), [&](void* y) {
      if (mine) {
        room = at::empty({bytes}, Q->options().dtype(at::kByte));
        ws = room.data_ptr();
      }
      return f_tree_fp4(q.p, k.p, v.p, c.Kc, c.Ks, c.Vc, c.Vs, (const int*)pos, (const int*)len, (const int*)start, (const int*)parent, (const int*)nodes, (const float*)slope, y, (float*)lse, ws, bytes,
                        c.M, c.B, T, c.C, heads, c.kv, c.d, q.model, q.row, k.model, k.row, scale, cap, dt, s);
    });
  });
}

// logits, token, k, vocab, nodes, scale, cap, out, workspace, device, stream: the tuple given, or a new one
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    at::ScalarType st;
    int device, M, N, V, k, B = 1, m = 0;
    float scale, cap;
    void *token, *vocab, *nodes, *ws, *s, *to[4] = {nullptr, nullptr, nullptr, nullptr};
    if (n != 11 || !types(a[0], a[9], &st, &device) || !whole(a[2], &k) || k < 0 || k > 32 || !number(a[5], &scale) || !number(a[6], &cap) || !stream_of(a[10], &s)) return not_taken();
    const at::Tensor* X = strided(a[0], st, device);
    if (!X || X->dim() != 3 || !size(X->size(0), &M) || !size(X->size(1), &N) || !size(X->size(2), &V) || M <= 0 || N <= 0 || V <= 0) return not_taken();
    Rows x;
    if (!rows(X, M, N, V, &x)) return not_taken();
    if (a[4] != Py_None) {
      const at::Tensor* t = strided(a[4], at::kInt, device);
      if (!t || t->dim() != 2 || !size(t->size(1), &B) || B <= 0 || N % B) return not_taken();
    }
    if (a[1] != Py_None) {
      const at::Tensor* t = strided(a[1], at::kInt, device);
      if (!t || t->dim() != 3 || !size(t->size(2), &m) || m <= 0) return not_taken();
    }
    if (!dense(a[1], at::kInt, {M, N, m}, device, false, &token) || !dense(a[3], at::kInt, {M}, device, false, &vocab) || !dense(a[4], at::kInt, {M, B}, device, false, &nodes)) return not_taken();
    const at::DimVector shape[4] = {{M, N, m}, {M, N}, {M, N, k}, {M, N, k}};
    const at::ScalarType type[4] = {at::kFloat, at::kFloat, at::kInt, at::kFloat};
    const bool wanted[4] = {m > 0, true, k > 0, k > 0};
    const bool given = a[7] != Py_None;
    if (given) {
      if (!PyTuple_CheckExact(a[7]) || PyTuple_GET_SIZE(a[7]) != 4) return not_taken();
      for (int i = 0; i < 4; ++i)
        if (!dense(PyTuple_GET_ITEM(a[7], i), type[i], shape[i], device, wanted[i], &to[i])) return not_taken();
    }
    long long bytes = f_logprobs_workspace(M, B, N / B, V, k);
    if (bytes < 0 || !workspace(a[8], device, &ws, &bytes)) return not_taken();
    const nf_dtype dt = type_of(*X);
    at::Tensor room, made[4];
    nf_status done_as;
    {
      Unlocked unlocked;
      if (a[8] == Py_None) {
        room = at::empty({bytes}, X->options().dtype(at::kByte));
        ws = room.data_ptr();
      }
      for (int i = 0; i < 4 && !given; ++i)
        if (wanted[i]) {
          made[i] = at::empty(shape[i], X->options().dtype(type[i]));
          to[i] = made[i].data_ptr();
        }
      done_as = f_logprobs(x.p, (const int*)token, (const int*)vocab, (const int*)nodes, (float*)to[0], (float*)to[1], (int*)to[2], (float*)to[3], ws, bytes, M, B, N / B, V, m, k, x.model, x.row, scale,
                           cap, dt, s);
    }
    at::Tensor none;
    PyObject* ok = done("netfuse_token_logprobs", done_as, given ? a[7] : Py_True, none);
    if (!ok || given) return ok;
    Py_DECREF(ok);
    PyObject* all = PyTuple_New(4);
    for (int i = 0; all && i < 4; ++i) {
      PyObject* t = Py_None;
      if (wanted[i]) t = THPVariable_Wrap(std::move(made[i]));
      else Py_INCREF(t);
      if (!t) {
        Py_DECREF(all);
        return nullptr;
      }
      PyTuple_SET_ITEM(all, i, t);
    }
    return all;
  });
}

// bind_step: the addresses of rotate_heads, cache_append_fp4, cache_read_fp4, attention_tree_fp4 and its workspace, token_logprobs and its workspace
PyObject* bind_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind_step takes seven addresses");
    return nullptr;
  }
  void* p[7];
  for (int i = 0; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  f_rotate = (decltype(f_rotate))p[0];
  f_append_fp4 = (decltype(f_append_fp4))p[1];
  f_read_fp4 = (decltype(f_read_fp4))p[2];
  f_tree_fp4 = (decltype(f_tree_fp4))p[3];
  f_tree_fp4_workspace = (decltype(f_tree_fp4_workspace))p[4];
  f_logprobs = (decltype(f_logprobs))p[5];
  f_logprobs_workspace = (decltype(f_logprobs_workspace))p[6];
  Py_RETURN_NONE;
}

// bind_decoder: the addresses of prompt, tree and its workspace, append, weigh, evict and its workspace
PyObject* bind_decoder(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind_decoder takes seven addresses");
    return nullptr;
  }
  void* p[7];
  for (int i = 0; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  f_prompt = (decltype(f_prompt))p[0];
  f_tree = (decltype(f_tree))p[1];
  f_tree_workspace = (decltype(f_tree_workspace))p[2];
  f_append = (decltype(f_append))p[3];
  f_weigh = (decltype(f_weigh))p[4];
  f_evict = (decltype(f_evict))p[5];
  f_evict_workspace = (decltype(f_evict_workspace))p[6];
  Py_RETURN_NONE;
}

// bind(error, linear, linear_packed, layernorm, attention, attention_relpos, conv2d): the addresses of the entry points
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind takes a callable and six addresses");
    return nullptr;
  }
  void* p[7];
  for (int i = 1; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Py_INCREF(a[0]);
  Py_XSETREF(g_error, a[0]);
  f_linear = (decltype(f_linear))p[1];
  f_packed = (decltype(f_packed))p[2];
  f_layernorm = (decltype(f_layernorm))p[3];
  f_attention = (decltype(f_attention))p[4];
  f_relpos = (decltype(f_relpos))p[5];
  f_conv2d = (decltype(f_conv2d))p[6];
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind), FAST(linear), FAST(linear_packed), FAST(layernorm), FAST(attention_packed), FAST(attention_relpos_packed),
                         FAST(conv2d), FAST(bind_decoder), FAST(attention_prompt), FAST(attention_tree), FAST(cache_append), FAST(cache_weigh), FAST(cache_evict), FAST(bind_step),
                         FAST(rotate_heads), FAST(cache_append_fp4), FAST(cache_read_fp4), FAST(attention_tree_fp4), FAST(token_logprobs), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the Python and torch whose headers are compiled in; the package uses the module with no other.
PyMODINIT_FUNC PyInit__binding() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", NETFUSE_BUILT_FOR) < 0) Py_CLEAR(m);
  return m;
}
