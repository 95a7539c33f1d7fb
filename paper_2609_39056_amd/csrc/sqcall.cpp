// Native argument marshalling of the Python binding's hot calls.
//
// binding.py describes each call with ctypes structures, which costs 7-8 us of
// Python per linear (nine tensors checked one attribute at a time, two
// structures, ten converted arguments): more than the two kernels of a small
// layer take.  The functions here read the same tensors through torch's C++
// interface and call the C ABI entry whose address the binding passes, with the
// interpreter lock released as ctypes releases it.
//
// They only take the plain case: exact torch.Tensor objects on the GPU,
// contiguous, exact ActParams / Weight objects, ints.  For anything else
// they return NotImplemented and the binding goes on with its ctypes path,
// which accepts or refuses the arguments as it always has.  No C++ exception
// leaves them.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <exception>
#include <initializer_list>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sq.h"

namespace {

PyObject* g_act_type = nullptr;     // binding.ActParams
PyObject* g_weight_type = nullptr;  // binding.Weight
PyObject* g_cache_type = nullptr;   // binding.KVCache
PyObject* g_rope_type = nullptr;    // binding.RopeParams
PyObject* s_tok2stream;
PyObject* s_gamma;
PyObject* s_clip;
PyObject* s_dinv;
PyObject* s_step;
PyObject* s_range_mode;
PyObject* s_act_bits;
PyObject* s_qw;
PyObject* s_w_scale;
PyObject* s_bias;
PyObject* s_w_group;
PyObject* s_cuda_stream;
PyObject* s_k;
PyObject* s_v;
PyObject* s_q_weight;
PyObject* s_k_weight;
PyObject* s_eps;
PyObject* s_cos;
PyObject* s_sin;
PyObject* s_interleaved;

// The readers return whether the argument is plain.  They refuse without an
// exception: throwing one took 3-6 us, which a call that goes on to the ctypes
// path (13 us) would pay on top.

// An owned attribute of `o`; null, with a Python error set, if there is none.
struct Attr {
  PyObject* p;
  Attr(PyObject* o, PyObject* name) : p(PyObject_GetAttr(o, name)) {}
  ~Attr() { Py_XDECREF(p); }
  Attr(const Attr&) = delete;
  Attr& operator=(const Attr&) = delete;
};

const at::Tensor* tensor(PyObject* o) {
  if (o == nullptr || !THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

template <typename T>
bool read(PyObject* o, T*& p) {
  const at::Tensor* t = tensor(o);
  if (t == nullptr) return false;
  p = static_cast<T*>(t->data_ptr());
  return true;
}
template <typename T>
bool read_or_null(PyObject* o, T*& p) {
  p = nullptr;
  return o == Py_None || read(o, p);
}

// A buffer and its size.
bool read(PyObject* o, void*& p, size_t& bytes) {
  if (!read(o, p)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  bytes = static_cast<size_t>(t.numel()) * t.element_size();
  return true;
}
bool read_or_null(PyObject* o, void*& p, size_t& bytes) {
  p = nullptr;
  bytes = 0;
  return o == Py_None || read(o, p, bytes);
}

bool read_int(PyObject* o, int32_t& v) {
  if (o == nullptr || !PyLong_Check(o)) return false;
  const long w = PyLong_AsLong(o);
  v = static_cast<int32_t>(w);
  return w == v && !(w == -1 && PyErr_Occurred());
}

bool size32(int64_t w, int32_t& v) {
  v = static_cast<int32_t>(w);
  return w == v;
}

// A matrix and its number of rows.
template <typename T>
bool read_rows(PyObject* o, T*& p, int32_t& rows) {
  if (!read(o, p)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.dim() >= 1 && size32(t.size(0), rows);
}

bool read_stream(PyObject* o, hipStream_t& s) {
  if (o == Py_None) {
    s = c10::hip::getCurrentHIPStream().stream();
    return true;
  }
  void* v;
  if (PyLong_CheckExact(o)) {
    v = PyLong_AsVoidPtr(o);
  } else {
    Attr a(o, s_cuda_stream);
    if (a.p == nullptr) return false;
    v = PyLong_AsVoidPtr(a.p);
  }
  s = static_cast<hipStream_t>(v);
  return v != nullptr || !PyErr_Occurred();
}

bool read(PyObject* o, sq_act_params& s) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_act_type) return false;
  Attr t2s(o, s_tok2stream), gamma(o, s_gamma), clip(o, s_clip), dinv(o, s_dinv), step(o, s_step),
      mode(o, s_range_mode), bits(o, s_act_bits);
  const at::Tensor* g = tensor(gamma.p);
  if (g == nullptr || g->dim() != 2) return false;
  s.gamma = static_cast<const float*>(g->data_ptr());
  return read_or_null(t2s.p, s.tok2stream) && read_or_null(clip.p, s.clip) && read_or_null(dinv.p, s.dinv) &&
         size32(g->size(1), s.num_streams) && size32(g->size(0), s.num_steps) && read_int(step.p, s.step) &&
         read_int(mode.p, s.range_mode) && read_int(bits.p, s.act_bits);
}

bool read(PyObject* o, sq_weight& s) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_weight_type) return false;
  Attr qw(o, s_qw), scale(o, s_w_scale), bias(o, s_bias), group(o, s_w_group);
  const at::Tensor* q = tensor(qw.p);
  if (q == nullptr || q->dim() < 2) return false;
  s.qw = static_cast<const uint8_t*>(q->data_ptr());
  return read_or_null(scale.p, s.w_scale) && read_or_null(bias.p, s.bias) && size32(q->size(0), s.N) &&
         size32(q->size(1) * 2, s.K) && read_int(group.p, s.w_group);
}

template <typename F>
bool read_entry(PyObject* address, F& fn) {
  void* p = PyLong_AsVoidPtr(address);
  fn = reinterpret_cast<F>(p);
  return p != nullptr;
}

// `args` reads the arguments (false: not plain; an exception of torch's counts as
// that), `call` makes the call.  The call runs without the interpreter lock and
// outside the try block: taking the lock back ends a daemon thread by a forced
// unwind once the interpreter shuts down, which no handler may catch (`...`
// would).
template <typename Args, typename Call>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, Args args, Call call) {
  if (n != want || g_act_type == nullptr) Py_RETURN_NOTIMPLEMENTED;
  bool plain = false;
  try {
    plain = args();
  } catch (const std::exception&) {
  }
  if (!plain) {
    PyErr_Clear();
    Py_RETURN_NOTIMPLEMENTED;
  }
  PyThreadState* save = PyEval_SaveThread();
  const sq_status st = call();
  PyEval_RestoreThread(save);
  return PyLong_FromLong(st);
}

// setup(ActParams, Weight)
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "setup(ActParams, Weight)");
    return nullptr;
  }
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XDECREF(g_act_type);
  Py_XDECREF(g_weight_type);
  g_act_type = a[0];
  g_weight_type = a[1];
  Py_RETURN_NONE;
}

// linear(address, x, act, w, y, out_dtype, workspace, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_linear_w4a8) fn;
  sq_act_params act;
  sq_weight w;
  const uint16_t* x;
  int32_t M, out;
  void *y, *ws;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 8,
      [&] {
        return read_entry(a[0], fn) && read_rows(a[1], x, M) && read(a[2], act) && read(a[3], w) && read(a[4], y) &&
               read_int(a[5], out) && read(a[6], ws, wb) && read_stream(a[7], s);
      },
      [&] { return fn(x, M, &act, &w, y, out, ws, wb, s); });
}

// gemm8(address, qx, row_scale, w, y, out_dtype, workspace, stream)
PyObject* gemm8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_gemm_w4a8) fn;
  sq_weight w;
  const int8_t* qx;
  const float* r;
  int32_t M, out;
  void *y, *ws;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 8,
      [&] {
        return read_entry(a[0], fn) && read_rows(a[1], qx, M) && read(a[2], r) && read(a[3], w) && read(a[4], y) &&
               read_int(a[5], out) && read_or_null(a[6], ws, wb) && read_stream(a[7], s);
      },
      [&] { return fn(qx, r, M, &w, y, out, ws, wb, s); });
}

// gemm4(address, qx, group_scale, act, w, y, out_dtype, workspace, stream)
PyObject* gemm4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_gemm_w4a4) fn;
  sq_act_params act;
  sq_weight w;
  const uint8_t* qx;
  const uint16_t* g;
  int32_t M, out;
  void *y, *ws;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 9,
      [&] {
        return read_entry(a[0], fn) && read_rows(a[1], qx, M) && read(a[2], g) && read(a[3], act) && read(a[4], w) &&
               read(a[5], y) && read_int(a[6], out) && read_or_null(a[7], ws, wb) && read_stream(a[8], s);
      },
      [&] { return fn(qx, g, M, &act, &w, y, out, ws, wb, s); });
}

// gemm4_fp8(address, qx, group_scale, kc, act, w, y, out_dtype, workspace, stream)
PyObject* gemm4_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_gemm_w4a4_fp8) fn;
  sq_act_params act;
  sq_weight w;
  const uint8_t* qx;
  const float *g, *kc;
  int32_t M, out;
  void *y, *ws;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 10,
      [&] {
        return read_entry(a[0], fn) && read_rows(a[1], qx, M) && read(a[2], g) && read(a[3], kc) && read(a[4], act) &&
               read(a[5], w) && read(a[6], y) && read_int(a[7], out) && read_or_null(a[8], ws, wb) &&
               read_stream(a[9], s);
      },
      [&] { return fn(qx, g, kc, M, &act, &w, y, out, ws, wb, s); });
}

// gelu8(address, x, act, w, act_next, qx_next, r_next, workspace, stream)
PyObject* gelu8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_linear_w4a8_gelu_quant) fn;
  sq_act_params act, next;
  sq_weight w;
  const uint16_t* x;
  int8_t* qx;
  float* r;
  int32_t M;
  void* ws;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 9,
      [&] {
        return read_entry(a[0], fn) && read_rows(a[1], x, M) && read(a[2], act) && read(a[3], w) && read(a[4], next) &&
               read(a[5], qx) && read(a[6], r) && read(a[7], ws, wb) && read_stream(a[8], s);
      },
      [&] { return fn(x, M, &act, &w, &next, qx, r, ws, wb, s); });
}

// gelu4(address, x, act, w, act_next, qx_next, scale_next, kc_next, workspace, stream)
PyObject* gelu4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_linear_w4a4_gelu_quant) fn;
  sq_act_params act, next;
  sq_weight w;
  const uint16_t* x;
  float* kc;
  int32_t M;
  void *qx, *sc, *ws;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 10,
      [&] {
        return read_entry(a[0], fn) && read_rows(a[1], x, M) && read(a[2], act) && read(a[3], w) && read(a[4], next) &&
               read(a[5], qx) && read(a[6], sc) && read_or_null(a[7], kc) && read(a[8], ws, wb) &&
               read_stream(a[9], s);
      },
      [&] { return fn(x, M, &act, &w, &next, qx, sc, kc, ws, wb, s); });
}

// quantize(address, x, act, qx, act_scale, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_quantize_act) fn;
  sq_act_params act;
  int32_t M, K;
  void *qx, *sc;
  hipStream_t s;
  const uint16_t* x;
  return guarded(
      n, 6,
      [&] {
        const at::Tensor* t = tensor(a[1]);
        return t != nullptr && t->dim() == 2 && size32(t->size(1), K) && read_entry(a[0], fn) &&
               read_rows(a[1], x, M) && read(a[2], act) && read(a[3], qx) && read(a[4], sc) && read_stream(a[5], s);
      },
      [&] { return fn(x, M, K, &act, qx, sc, s); });
}

// ------------------------------------------------------------------ the token step
// Its binding functions check sizes and types as well: what does not pass here
// is refused by the ctypes path.

bool half(at::ScalarType t) { return t == at::kBFloat16 || t == at::kHalf; }
int32_t half_code(at::ScalarType t) { return t == at::kBFloat16 ? SQ_OUT_BF16 : SQ_OUT_F16; }
bool is_out(at::ScalarType t, int32_t code) {
  return (code == SQ_OUT_F32 && t == at::kFloat) || (code == SQ_OUT_BF16 && t == at::kBFloat16) ||
         (code == SQ_OUT_F16 && t == at::kHalf);
}

bool read_float(PyObject* o, float& v) {
  if (o == nullptr || !PyFloat_CheckExact(o)) return false;
  v = static_cast<float>(PyFloat_AS_DOUBLE(o));
  return true;
}

// A contiguous tensor of a type and of the given sizes (-1: any).
template <typename T>
bool read_sized(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> sizes, T*& p) {
  const at::Tensor* t = tensor(o);
  if (t == nullptr || t->scalar_type() != type || t->dim() != static_cast<int64_t>(sizes.size())) return false;
  int64_t d = 0;
  for (const int64_t n : sizes) {
    if (n >= 0 && t->size(d) != n) return false;
    ++d;
  }
  p = static_cast<T*>(t->data_ptr());
  return true;
}
template <typename T>
bool read_sized_or_null(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> sizes, T*& p) {
  p = nullptr;
  return o == Py_None || read_sized(o, type, sizes, p);
}

// [T, heads, D], a token's heads contiguous.
bool read_heads(PyObject* o, at::ScalarType type, int64_t T, int64_t D, const void*& p, int64_t& stride, int32_t& heads) {
  if (o == nullptr || !THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != type || t.dim() != 3 || t.size(0) != T || t.size(2) != D ||
      t.stride(2) != 1 || (t.size(1) > 1 && t.stride(1) != D))
    return false;
  p = t.data_ptr();
  stride = T > 1 ? t.stride(0) : t.size(1) * D;
  return size32(t.size(1), heads);
}

bool read(PyObject* o, sq_kv_cache& c, at::ScalarType& type) {
  if (o == nullptr || reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_cache_type) return false;
  Attr ka(o, s_k), va(o, s_v);
  const at::Tensor *k = tensor(ka.p), *v = tensor(va.p);
  if (k == nullptr || v == nullptr || k->dim() != 4 || !half(k->scalar_type()) || v->scalar_type() != k->scalar_type() ||
      v->sizes() != k->sizes())
    return false;
  type = k->scalar_type();
  c.k = k->data_ptr();
  c.v = v->data_ptr();
  c.dtype = half_code(type);
  return size32(k->size(0), c.num_pages) && size32(k->size(1), c.num_heads) && size32(k->size(2), c.page_size) &&
         size32(k->size(3), c.head_dim);
}

bool read(PyObject* o, sq_rope_params& p, int64_t D) {
  if (o == nullptr || reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_rope_type) return false;
  Attr qw(o, s_q_weight), kw(o, s_k_weight), eps(o, s_eps), cos(o, s_cos), sin(o, s_sin), inter(o, s_interleaved);
  if (!read_sized_or_null(qw.p, at::kFloat, {D}, p.q_weight) || !read_sized_or_null(kw.p, at::kFloat, {D}, p.k_weight) ||
      !read_float(eps.p, p.eps) || inter.p == nullptr || !PyBool_Check(inter.p))
    return false;
  p.interleaved = inter.p == Py_True;
  p.cos = p.sin = nullptr;
  p.num_pos = p.rot_dim = 0;
  if (cos.p == Py_None && sin.p == Py_None) return true;
  const at::Tensor* c = tensor(cos.p);
  if (c == nullptr || c->dim() != 2 || c->scalar_type() != at::kFloat) return false;
  p.cos = static_cast<const float*>(c->data_ptr());
  return read_sized(sin.p, at::kFloat, {c->size(0), c->size(1)}, p.sin) && size32(c->size(0), p.num_pos) &&
         size32(2 * c->size(1), p.rot_dim);
}

// setup_token(KVCache, RopeParams)
PyObject* setup_token(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "setup_token(KVCache, RopeParams)");
    return nullptr;
  }
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XDECREF(g_cache_type);
  Py_XDECREF(g_rope_type);
  g_cache_type = a[0];
  g_rope_type = a[1];
  Py_RETURN_NONE;
}

// kv_plan(address, cached_len, new_len, page_size, free_pages, free_head, table, slot, pos, token_start, kv_len,
//         free_head_out, stream)
PyObject* kv_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_kv_plan) fn;
  const int32_t *cached, *fresh, *free_pages, *head;
  int32_t *table, *slot, *pos, *start, *kv_len, *head_out;
  int32_t R, page, num_free, max_pages, max_tokens;
  hipStream_t s;
  return guarded(
      n, 13,
      [&] {
        if (!read_entry(a[0], fn) || !read_sized(a[6], at::kInt, {-1, -1}, table) ||
            !read_sized(a[4], at::kInt, {-1}, free_pages) || !read_sized(a[7], at::kInt, {-1}, slot))
          return false;
        const at::Tensor& t = THPVariable_Unpack(a[6]);
        return size32(t.size(0), R) && size32(t.size(1), max_pages) &&
               size32(THPVariable_Unpack(a[4]).size(0), num_free) && size32(THPVariable_Unpack(a[7]).size(0), max_tokens) &&
               read_sized(a[1], at::kInt, {R}, cached) && read_sized(a[2], at::kInt, {R}, fresh) && read_int(a[3], page) &&
               read_sized_or_null(a[5], at::kInt, {1}, head) && read_sized(a[8], at::kInt, {max_tokens}, pos) &&
               read_sized(a[9], at::kInt, {int64_t{R} + 1}, start) && read_sized(a[10], at::kInt, {R}, kv_len) &&
               read_sized(a[11], at::kInt, {1}, head_out) && read_stream(a[12], s);
      },
      [&] {
        return fn(cached, fresh, R, page, free_pages, num_free, head, table, max_pages, max_tokens, slot, pos, start,
                  kv_len, head_out, s);
      });
}

// rope(address, q, k, v, params, pos, slot, q_out, k_out, kv, stream)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_qk_norm_rope) fn;
  const void *q, *k, *v = nullptr;
  int64_t qs, ks, vs = 0;
  int32_t T, Hq, Hk, Hv, D, dtype;
  sq_rope_params p;
  sq_kv_cache c;
  bool has_cache;
  const int32_t *pos, *slot;
  void *q_out, *k_out;
  hipStream_t s;
  return guarded(
      n, 11,
      [&] {
        if (!read_entry(a[0], fn) || a[1] == nullptr || !THPVariable_CheckExact(a[1])) return false;
        const at::Tensor& t = THPVariable_Unpack(a[1]);
        if (t.dim() != 3 || !half(t.scalar_type()) || !size32(t.size(0), T) || !size32(t.size(2), D)) return false;
        const at::ScalarType type = t.scalar_type();
        at::ScalarType cache_type;
        dtype = half_code(type);
        has_cache = a[9] != Py_None;
        return read_heads(a[1], type, T, D, q, qs, Hq) && read_heads(a[2], type, T, D, k, ks, Hk) &&
               (a[3] == Py_None || (read_heads(a[3], type, T, D, v, vs, Hv) && Hv == Hk)) && read(a[4], p, D) &&
               read_sized_or_null(a[5], at::kInt, {T}, pos) && read_sized_or_null(a[6], at::kInt, {T}, slot) &&
               read_sized(a[7], type, {T, Hq, D}, q_out) && read_sized_or_null(a[8], type, {T, Hk, D}, k_out) &&
               (!has_cache || read(a[9], c, cache_type)) && read_stream(a[10], s);
      },
      [&] {
        return fn(q, qs, k, ks, v, vs, T, Hq, Hk, D, dtype, &p, pos, slot, q_out, k_out, has_cache ? &c : nullptr, s);
      });
}

// attn(address, q, kv, table, kv_len, max_kv_len, window, scale, out, out_dtype, lse, workspace, stream)
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_attn_paged) fn;
  const void* q;
  int64_t qs;
  sq_kv_cache c;
  const int32_t *table, *kv_len;
  int32_t R, Hq, max_pages, longest, window, out_dtype;
  float scale;
  void *out, *ws;
  float* lse;
  size_t wb;
  hipStream_t s;
  return guarded(
      n, 13,
      [&] {
        at::ScalarType type;
        if (!read_entry(a[0], fn) || !read(a[2], c, type) || !read_sized(a[3], at::kInt, {-1, -1}, table)) return false;
        const at::Tensor& t = THPVariable_Unpack(a[3]);
        if (!size32(t.size(0), R) || !size32(t.size(1), max_pages) || !read_heads(a[1], type, R, c.head_dim, q, qs, Hq) ||
            !read_int(a[9], out_dtype))
          return false;
        const at::Tensor* o = tensor(a[8]);
        if (o == nullptr || !is_out(o->scalar_type(), out_dtype)) return false;
        return read_sized(a[8], o->scalar_type(), {R, Hq, c.head_dim}, out) && read_sized(a[4], at::kInt, {R}, kv_len) &&
               read_int(a[5], longest) && read_int(a[6], window) && read_float(a[7], scale) &&
               read_sized_or_null(a[10], at::kFloat, {R, Hq}, lse) && read(a[11], ws, wb) && read_stream(a[12], s);
      },
      [&] {
        return fn(q, qs, R, Hq, &c, table, max_pages, kv_len, longest, window, scale, out, out_dtype, lse, ws, wb, s);
      });
}

// linear16(address, x, dinv, w, y, out_dtype, stream)
PyObject* linear16(PyObject*, PyObject* const* a, Py_ssize_t n) {
  decltype(&sq_linear_w4a16) fn;
  const uint16_t* x;
  const float* dinv;
  sq_weight w;
  void* y;
  int32_t M, out;
  hipStream_t s;
  return guarded(
      n, 7,
      [&] {
        if (!read_entry(a[0], fn) || !read(a[3], w) || !read_sized(a[1], at::kBFloat16, {-1, w.K}, x) ||
            !size32(THPVariable_Unpack(a[1]).size(0), M) || !read_int(a[5], out))
          return false;
        const at::Tensor* o = tensor(a[4]);
        return o != nullptr && is_out(o->scalar_type(), out) && read_sized(a[4], o->scalar_type(), {M, w.N}, y) &&
               read_sized_or_null(a[2], at::kFloat, {w.K}, dinv) && read_stream(a[6], s);
      },
      [&] { return fn(x, M, dinv, &w, y, out, s); });
}

PyMethodDef methods[] = {
    {"setup_token", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(setup_token)), METH_FASTCALL, nullptr},
    {"kv_plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_plan)), METH_FASTCALL, nullptr},
    {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rope)), METH_FASTCALL, nullptr},
    {"attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attn)), METH_FASTCALL, nullptr},
    {"linear16", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear16)), METH_FASTCALL, nullptr},
    {"setup", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(setup)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"gemm8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gemm8)), METH_FASTCALL, nullptr},
    {"gemm4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gemm4)), METH_FASTCALL, nullptr},
    {"gemm4_fp8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gemm4_fp8)), METH_FASTCALL, nullptr},
    {"gelu8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gelu8)), METH_FASTCALL, nullptr},
    {"gelu4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gelu4)), METH_FASTCALL, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "sqcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_sqcall(void) {
  s_tok2stream = PyUnicode_InternFromString("tok2stream");
  s_gamma = PyUnicode_InternFromString("gamma");
  s_clip = PyUnicode_InternFromString("clip");
  s_dinv = PyUnicode_InternFromString("dinv");
  s_step = PyUnicode_InternFromString("step");
  s_range_mode = PyUnicode_InternFromString("range_mode");
  s_act_bits = PyUnicode_InternFromString("act_bits");
  s_qw = PyUnicode_InternFromString("qw");
  s_w_scale = PyUnicode_InternFromString("w_scale");
  s_bias = PyUnicode_InternFromString("bias");
  s_w_group = PyUnicode_InternFromString("w_group");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_k = PyUnicode_InternFromString("k");
  s_v = PyUnicode_InternFromString("v");
  s_q_weight = PyUnicode_InternFromString("q_weight");
  s_k_weight = PyUnicode_InternFromString("k_weight");
  s_eps = PyUnicode_InternFromString("eps");
  s_cos = PyUnicode_InternFromString("cos");
  s_sin = PyUnicode_InternFromString("sin");
  s_interleaved = PyUnicode_InternFromString("interleaved");
  PyObject* m = PyModule_Create(&module_def);
  if (m != nullptr && PyModule_AddStringConstant(m, "built_for", SQCALL_BUILT_FOR) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
