// The host side of the binding's frequent calls: allocation of the outputs and the call of the C entry point, without the
// Python objects in between.  A host-bound program (small operands, the decode stage) spends its time here: a torch.empty takes
// 1.4 us from Python and 0.3 from here, the marshalling of ten arguments through ctypes 0.7; us a call, host-bound, before -> now:
// quantize of 16 x 256 10.3 -> 4.4, dequantize 7.2 -> 3.9, gemm_bf16a of 8 x 4096 x 4096 (two launches) 13.0 -> 6.3.  About 3 us
// of each is a kernel launch.
//
// Every function takes the common case only and returns None for anything else -- another tensor type, layout or dtype, an argument
// that the C entry point refuses -- before it has launched anything; the caller then goes through its general code, which raises.
#include <torch/extension.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/hip/HIPStream.h>
#include <cstdint>
#include "mxp.h"

namespace {

struct Entry {
  decltype(&mxp_quantize) quantize;
  decltype(&mxp_dequantize) dequantize;
  decltype(&mxp_gemm) gemm;
  decltype(&mxp_gemm_workspace_bytes_fmt) gemm_ws;
  decltype(&mxp_gemm_bf16a) bf16a;
  decltype(&mxp_gemm_bf16a_workspace_bytes) bf16a_ws;
  decltype(&mxp_gemm_decode_bf16a) decode_bf16a;
  decltype(&mxp_gemm_w4a16_ws) w4a16;
  decltype(&mxp_gemm_w4a16_workspace_bytes) w4a16_ws;
  decltype(&mxp_rmsnorm_quantize) rmsnorm_quantize;
  decltype(&mxp_cache_bytes) cache_bytes;
  decltype(&mxp_cache_write) cache_write;
  decltype(&mxp_cache_read) cache_read;
  decltype(&mxp_attention) attention;
  decltype(&mxp_attention_workspace_bytes) attention_ws;
} lib = {};

// a plain CUDA tensor, or nullptr
const at::Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() ? &t : nullptr;
}
// fp32 / bf16 rows with unit inner stride: the dtype code, or -1
int rows_dtype(const at::Tensor* t) {
  if (!t || t->dim() != 2 || t->stride(1) != 1) return -1;
  return t->scalar_type() == at::kFloat ? MXP_F32 : t->scalar_type() == at::kBFloat16 ? MXP_BF16 : -1;
}
int64_t ld(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.size(1), 1); }
int64_t code_bits(int64_t fmt) { return fmt < MXP_FMT_MXFP6 ? 4 : fmt < MXP_FMT_MXFP8 ? 6 : 8; }

struct Quantized {                                           // (elems, scales, idx), idx possibly None
  const at::Tensor *el = nullptr, *sc = nullptr;
  uint8_t* ix = nullptr;
  bool take(PyObject* q) {
    if (!PyTuple_CheckExact(q) || PyTuple_GET_SIZE(q) != 3) return false;
    el = tensor(PyTuple_GET_ITEM(q, 0));
    sc = tensor(PyTuple_GET_ITEM(q, 1));
    if (!el || !sc || el->dim() != 2 || sc->dim() != 2) return false;
    PyObject* i = PyTuple_GET_ITEM(q, 2);
    if (i == Py_None) return true;
    const at::Tensor* t = tensor(i);
    if (t) ix = static_cast<uint8_t*>(t->data_ptr());
    return t != nullptr;
  }
  const uint8_t* e() const { return static_cast<const uint8_t*>(el->data_ptr()); }
  const uint8_t* s() const { return static_cast<const uint8_t*>(sc->data_ptr()); }
};

at::Tensor bytes(const at::Tensor& like, at::IntArrayRef size) { return at::empty(size, at::TensorOptions().dtype(at::kByte).device(like.device())); }
at::Tensor output(const at::Tensor& like, int64_t M, int64_t N, int64_t d) {
  return at::empty({M, N}, at::TensorOptions().dtype(d == MXP_BF16 ? at::kBFloat16 : at::kFloat).device(like.device()));
}
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }
int64_t integer(PyObject* o) { return PyLong_AsLongLong(o); }

// `n` arguments, those from `first` on integers of 64 bits (a longer one would leave an error set)
bool arguments(PyObject* const* a, Py_ssize_t given, Py_ssize_t n, Py_ssize_t first) {
  if (given != n) return false;
  for (Py_ssize_t i = first; i < n; ++i) {
    int overflow = 0;
    if (!PyLong_CheckExact(a[i]) || (PyLong_AsLongLongAndOverflow(a[i], &overflow), overflow != 0)) return false;
  }
  return true;
}
template <class F>
int unlocked(F&& f) {
  pybind11::gil_scoped_release release;
  return f();
}

PyObject* fast_init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void** slots = reinterpret_cast<void**>(&lib);
  if (n != (Py_ssize_t)(sizeof(lib) / sizeof(void*))) {
    PyErr_SetString(PyExc_TypeError, "one address per entry point");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) slots[i] = PyLong_AsVoidPtr(a[i]);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyObject* fast_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // x, fmt
  HANDLE_TH_ERRORS
  const at::Tensor* x = arguments(a, n, 2, 1) ? tensor(a[0]) : nullptr;
  const int dt = rows_dtype(x);
  if (dt < 0) Py_RETURN_NONE;
  const int64_t rows = x->size(0), K = x->size(1), fmt = integer(a[1]);
  if (K % 32 != 0 || fmt < MXP_FMT_MXFP4 || fmt > MXP_FMT_MXFP8P) Py_RETURN_NONE;
  at::Tensor e = bytes(*x, {rows, K * code_bits(fmt) / 8}), s = bytes(*x, {rows, K / 32}), i = bytes(*x, {rows, K / 32});
  if (unlocked([&] {
        return lib.quantize(x->data_ptr(), dt, rows, K, ld(*x), (int)fmt, static_cast<uint8_t*>(e.data_ptr()), static_cast<uint8_t*>(s.data_ptr()),
                            static_cast<uint8_t*>(i.data_ptr()), stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  PyObject* out = PyTuple_New(3);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(e)));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(s)));
  PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(std::move(i)));
  return out;
  END_HANDLE_TH_ERRORS
}

PyObject* fast_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // q, fmt, dtype code
  HANDLE_TH_ERRORS
  Quantized q;
  if (!arguments(a, n, 3, 1) || !q.take(a[0])) Py_RETURN_NONE;
  const int64_t fmt = integer(a[1]), d = integer(a[2]);
  if (fmt < MXP_FMT_MXFP4 || fmt > MXP_FMT_MXFP8P) Py_RETURN_NONE;
  const int64_t rows = q.el->size(0), K = q.el->size(1) * 8 / code_bits(fmt);
  at::Tensor out = output(*q.el, rows, K, d);
  if (unlocked([&] { return lib.dequantize(q.e(), q.s(), q.ix, (int)fmt, rows, K, out.data_ptr(), (int)d, std::max<int64_t>(K, 1), stream()); }) != MXP_OK)
    Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyObject* fast_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {   // qa, qb, fmt_a, fmt_b, dtype code
  HANDLE_TH_ERRORS
  Quantized qa, qb;
  if (!arguments(a, n, 5, 2) || !qa.take(a[0]) || !qb.take(a[1])) Py_RETURN_NONE;
  const int64_t fa = integer(a[2]), fb = integer(a[3]), d = integer(a[4]);
  const int64_t M = qa.el->size(0), K = qa.sc->size(1) * 32, N = qb.el->size(0);
  if (qb.sc->size(1) * 32 != K) Py_RETURN_NONE;
  at::Tensor out = output(*qa.el, M, N, d);
  at::Tensor ws = bytes(*qa.el, {std::max<int64_t>((int64_t)lib.gemm_ws(M, N, K, (int)fa, (int)fb), 16)});
  if (unlocked([&] {
        return lib.gemm(M, N, K, qa.e(), qa.s(), qa.ix, (int)fa, qb.e(), qb.s(), qb.ix, (int)fb, out.data_ptr(), (int)d, std::max<int64_t>(N, 1),
                        ws.data_ptr(), (size_t)ws.numel(), stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyObject* fast_gemm_bf16a(PyObject*, PyObject* const* a, Py_ssize_t n) {   // activations, image, fmt_a (not MXFP4++), N, dtype code, image kind
  HANDLE_TH_ERRORS
  if (!arguments(a, n, 6, 2)) Py_RETURN_NONE;
  const at::Tensor *x = tensor(a[0]), *img = tensor(a[1]);
  const int dt = rows_dtype(x);
  if (dt < 0 || !img) Py_RETURN_NONE;
  const int64_t fa = integer(a[2]), N = integer(a[3]), d = integer(a[4]), kind = integer(a[5]), M = x->size(0), K = x->size(1);
  if (N < 0 || K % 32 != 0) Py_RETURN_NONE;
  at::Tensor out = output(*x, M, N, d);
  at::Tensor ws = bytes(*x, {std::max<int64_t>((int64_t)lib.bf16a_ws(M, K), 16)});
  if (unlocked([&] {
        return lib.bf16a(M, N, K, x->data_ptr(), dt, ld(*x), (int)fa, img->data_ptr(), (int)kind, out.data_ptr(), (int)d, std::max<int64_t>(N, 1),
                         ws.data_ptr(), (size_t)ws.numel(), stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyObject* fast_gemm_decode_bf16a(PyObject*, PyObject* const* a, Py_ssize_t n) {   // activations, qw, fmt_a, fmt_w, dtype code
  HANDLE_TH_ERRORS
  Quantized w;
  if (!arguments(a, n, 5, 2) || !w.take(a[1])) Py_RETURN_NONE;
  const at::Tensor* x = tensor(a[0]);
  const int dt = rows_dtype(x);
  if (dt < 0) Py_RETURN_NONE;
  const int64_t fa = integer(a[2]), fw = integer(a[3]), d = integer(a[4]), M = x->size(0), K = x->size(1), N = w.el->size(0);
  if (K % 32 != 0) Py_RETURN_NONE;
  at::Tensor out = output(*x, M, N, d);
  at::Tensor ws = bytes(*x, {std::max<int64_t>((int64_t)lib.bf16a_ws(M, K), 16)});
  if (unlocked([&] {
        return lib.decode_bf16a(M, N, K, x->data_ptr(), dt, ld(*x), (int)fa, w.e(), w.s(), w.ix, (int)fw, out.data_ptr(), (int)d, std::max<int64_t>(N, 1),
                                ws.data_ptr(), (size_t)ws.numel(), stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyObject* fast_gemm_w4a16(PyObject*, PyObject* const* a, Py_ssize_t n) {   // activations, qw, fmt_w, dtype code
  HANDLE_TH_ERRORS
  Quantized w;
  if (!arguments(a, n, 4, 2) || !w.take(a[1])) Py_RETURN_NONE;
  const at::Tensor* x = tensor(a[0]);
  const int dt = rows_dtype(x);
  if (dt < 0) Py_RETURN_NONE;
  const int64_t fw = integer(a[2]), d = integer(a[3]), M = x->size(0), K = x->size(1), N = w.el->size(0);
  if (w.sc->size(1) * 32 != K) Py_RETURN_NONE;
  at::Tensor out = output(*x, M, N, d), ws;
  const int64_t need = (int64_t)lib.w4a16_ws(M, N, K, (int)fw);
  if (need > 0) {
    try {
      ws = bytes(*x, {need});
    } catch (const c10::OutOfMemoryError&) {                 // room that the call can do without
      ws = at::Tensor();
    }
  }
  if (unlocked([&] {
        return lib.w4a16(M, N, K, x->data_ptr(), dt, ld(*x), w.e(), w.s(), w.ix, (int)fw, out.data_ptr(), (int)d, std::max<int64_t>(N, 1),
                         ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? (size_t)need : 0, stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

// ---- norm, cache, attention: besides, every tensor lies on the current device and has the shape that the others say -----
bool here(const at::Tensor* t) { return t && t->device().index() == c10::hip::getCurrentHIPStream().device_index(); }
bool none_or_tensor(PyObject* o, const at::Tensor*& t) {
  t = o == Py_None ? nullptr : tensor(o);
  return o == Py_None || here(t);
}
void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
bool real(PyObject* o, float& v) {
  if (!PyFloat_CheckExact(o)) return false;
  v = (float)PyFloat_AS_DOUBLE(o);
  return true;
}
bool whole(const at::Tensor* t, at::ScalarType type, int64_t dims) { return here(t) && t->scalar_type() == type && t->dim() == dims && t->is_contiguous(); }
int dtype_code(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? MXP_F32 : t.scalar_type() == at::kBFloat16 ? MXP_BF16 : -1; }
// [rows][heads][D] without gaps inside a row
bool heads_of(const at::Tensor* t, int64_t rows, int64_t heads, int64_t D) {
  return here(t) && t->dim() == 3 && (rows < 0 || t->size(0) == rows) && (heads < 0 || t->size(1) == heads) && t->size(2) == D && t->stride(2) == 1 &&
         (t->size(1) == 1 || t->stride(1) == D) && dtype_code(*t) >= 0;
}
int64_t ld3(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.size(1) * t.size(2), 1); }

struct Cache {                                               // data, and page_tokens, kv_heads, head_dim, fmt
  const at::Tensor* t = nullptr;
  int64_t pages = 0, page = 0, heads = 0, D = 0, fmt = 0;
  bool take(PyObject* d, PyObject* const* geometry) {
    t = tensor(d);
    if (!whole(t, at::kByte, 4)) return false;
    pages = t->size(0);
    page = integer(geometry[0]);
    heads = integer(geometry[1]);
    D = integer(geometry[2]);
    fmt = integer(geometry[3]);
    return fmt >= 0 && fmt <= MXP_FMT_MXFP8P && t->numel() > 0 && t->size(1) == heads && (size_t)t->numel() == lib.cache_bytes(pages, page, heads, D, (int)fmt);
  }
};

PyObject* fast_rmsnorm_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // x, weight, residual or None, eps, fmt
  HANDLE_TH_ERRORS
  if (!arguments(a, n, 5, 4)) Py_RETURN_NONE;
  const at::Tensor *x = tensor(a[0]), *w = tensor(a[1]), *r = nullptr;
  const int dt = rows_dtype(x);
  float eps = 0;
  if (dt < 0 || !here(x) || !here(w) || !none_or_tensor(a[2], r) || !real(a[3], eps)) Py_RETURN_NONE;
  const int64_t rows = x->size(0), K = x->size(1), fmt = integer(a[4]);
  if (K % 32 != 0 || fmt < MXP_FMT_MXFP4 || fmt > MXP_FMT_MXFP8P || w->dim() != 1 || w->size(0) != K || w->stride(0) != 1 || dtype_code(*w) < 0) Py_RETURN_NONE;
  if (r && (rows_dtype(r) != dt || r->size(0) != rows || r->size(1) != K)) Py_RETURN_NONE;
  at::Tensor e = bytes(*x, {rows, K * code_bits(fmt) / 8}), s = bytes(*x, {rows, K / 32}), i = bytes(*x, {rows, K / 32}), h;
  if (r) h = output(*x, rows, K, dt);
  if (unlocked([&] {
        return lib.rmsnorm_quantize(x->data_ptr(), data(r), dt, rows, K, ld(*x), r ? ld(*r) : 0, w->data_ptr(), dtype_code(*w), eps,
                                    r ? h.data_ptr() : nullptr, r ? std::max<int64_t>(K, 1) : 0, (int)fmt, static_cast<uint8_t*>(e.data_ptr()),
                                    static_cast<uint8_t*>(s.data_ptr()), static_cast<uint8_t*>(i.data_ptr()), stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  PyObject *q = PyTuple_New(3), *out = PyTuple_New(2);
  if (!q || !out) {
    Py_XDECREF(q);
    Py_XDECREF(out);
    return nullptr;
  }
  PyTuple_SET_ITEM(q, 0, THPVariable_Wrap(std::move(e)));
  PyTuple_SET_ITEM(q, 1, THPVariable_Wrap(std::move(s)));
  PyTuple_SET_ITEM(q, 2, THPVariable_Wrap(std::move(i)));
  PyTuple_SET_ITEM(out, 0, q);
  if (!r) Py_INCREF(a[0]);
  PyTuple_SET_ITEM(out, 1, r ? THPVariable_Wrap(std::move(h)) : a[0]);
  return out;
  END_HANDLE_TH_ERRORS
}

PyObject* fast_cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {   // data, k, v, slots, page_tokens, kv_heads, head_dim, fmt
  HANDLE_TH_ERRORS
  Cache c;
  if (!arguments(a, n, 8, 4) || !c.take(a[0], a + 4)) Py_RETURN_NONE;
  const at::Tensor *k = tensor(a[1]), *v = tensor(a[2]), *slots = tensor(a[3]);
  if (!whole(slots, at::kLong, 1)) Py_RETURN_NONE;
  const int64_t tokens = slots->size(0);
  if (!heads_of(k, tokens, c.heads, c.D) || !heads_of(v, tokens, c.heads, c.D) || k->scalar_type() != v->scalar_type()) Py_RETURN_NONE;
  if (unlocked([&] {
        return lib.cache_write(k->data_ptr(), v->data_ptr(), dtype_code(*k), tokens, ld3(*k), ld3(*v), static_cast<const int64_t*>(slots->data_ptr()),
                               c.t->data_ptr(), c.pages, c.page, c.heads, c.D, (int)c.fmt, stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

PyObject* fast_cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {   // data, slots, page_tokens, kv_heads, head_dim, fmt, dtype code
  HANDLE_TH_ERRORS
  Cache c;
  if (!arguments(a, n, 7, 2) || !c.take(a[0], a + 2)) Py_RETURN_NONE;
  const at::Tensor* slots = tensor(a[1]);
  const int64_t d = integer(a[6]);
  if (!whole(slots, at::kLong, 1) || (d != MXP_F32 && d != MXP_BF16)) Py_RETURN_NONE;
  const int64_t tokens = slots->size(0);
  const auto opts = at::TensorOptions().dtype(d == MXP_BF16 ? at::kBFloat16 : at::kFloat).device(slots->device());
  at::Tensor k = at::empty({tokens, c.heads, c.D}, opts), v = at::empty({tokens, c.heads, c.D}, opts);
  if (unlocked([&] {
        return lib.cache_read(c.t->data_ptr(), c.pages, c.page, c.heads, c.D, (int)c.fmt, static_cast<const int64_t*>(slots->data_ptr()), tokens,
                              k.data_ptr(), v.data_ptr(), (int)d, c.heads * c.D, c.heads * c.D, stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(k)));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(v)));
  return out;
  END_HANDLE_TH_ERRORS
}

// q, data, table, kv_len, q_start or None, lse or None, scale, causal, window, max_q, max_kv (-1: left out), dtype code, page_tokens, kv_heads, head_dim, fmt
PyObject* fast_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Cache c;
  float scale = 0;
  const at::Tensor *start = nullptr, *lse = nullptr;
  if (!arguments(a, n, 16, 7) || !c.take(a[1], a + 12) || !none_or_tensor(a[4], start) || !none_or_tensor(a[5], lse) || !real(a[6], scale)) Py_RETURN_NONE;
  const at::Tensor *q = tensor(a[0]), *table = tensor(a[2]), *len = tensor(a[3]);
  const int64_t causal = integer(a[7]), window = integer(a[8]), d = integer(a[11]);
  int64_t max_q = integer(a[9]), max_kv = integer(a[10]);
  if (!heads_of(q, -1, -1, c.D) || !whole(len, at::kInt, 1) || !whole(table, at::kInt, 2) || (d != MXP_F32 && d != MXP_BF16)) Py_RETURN_NONE;
  const int64_t rows = q->size(0), heads = q->size(1), seqs = len->size(0);
  if (table->size(0) != seqs || (start && (!whole(start, at::kInt, 1) || start->size(0) != seqs + 1)) ||
      (lse && (!whole(lse, at::kFloat, 2) || lse->size(0) != rows || lse->size(1) != heads)))
    Py_RETURN_NONE;
  if (max_q < 0) max_q = start ? rows : 1;
  if (max_kv < 0) max_kv = std::min<int64_t>(table->size(1) * c.page, (int64_t)1 << 30);
  at::Tensor out = at::empty({rows, heads, c.D}, at::TensorOptions().dtype(d == MXP_BF16 ? at::kBFloat16 : at::kFloat).device(q->device())), ws;
  const int64_t need = (int64_t)lib.attention_ws(seqs, rows, max_q, max_kv, heads, c.heads, c.D, (int)causal, window);
  if (need > 0) ws = bytes(*q, {need});
  if (unlocked([&] {
        return lib.attention(q->data_ptr(), dtype_code(*q), ld3(*q), rows, heads, static_cast<const int32_t*>(data(start)), static_cast<const int32_t*>(len->data_ptr()),
                             static_cast<const int32_t*>(table->data_ptr()), table->size(1), seqs, max_q, max_kv, scale, (int)causal, window, c.t->data_ptr(),
                             c.pages, c.page, c.heads, c.D, (int)c.fmt, out.data_ptr(), (int)d, heads * c.D, static_cast<float*>(data(lse)),
                             need > 0 ? ws.data_ptr() : nullptr, (size_t)std::max<int64_t>(need, 0), stream());
      }) != MXP_OK)
    Py_RETURN_NONE;
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

#define MXP_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fast_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MXP_METHOD(init),      MXP_METHOD(quantize),          MXP_METHOD(dequantize), MXP_METHOD(gemm),
                         MXP_METHOD(gemm_bf16a), MXP_METHOD(gemm_decode_bf16a), MXP_METHOD(gemm_w4a16),
                         MXP_METHOD(rmsnorm_quantize), MXP_METHOD(cache_write), MXP_METHOD(cache_read), MXP_METHOD(attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mxp_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mxp_binding() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", MXP_TORCH_VERSION) != 0) Py_CLEAR(m);   // of the headers it was compiled with
  return m;
}
