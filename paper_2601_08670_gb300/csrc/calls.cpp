// calls.cpp -- the calls over paged caches and on logits for the Python binding: a
// CPython module that checks the tensors (types, shapes, strides, device), takes
// their addresses and calls the C ABI.  The checks alone took 3 to 6 us a call in
// Python, beside 3 us for the call itself; a call that a program makes for every
// layer and token is mostly that.  No arithmetic is done here.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <stdexcept>
#include <string>

#include "pced.h"

namespace {

struct Refused : std::runtime_error {  // becomes ValueError
  using std::runtime_error::runtime_error;
};

void require(bool ok, const char* what) {
  if (!ok) throw Refused(what);
}

// a tensor argument, null for None
const at::Tensor* tensor(PyObject* o, const char* what) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw Refused(std::string(what) + ": a tensor");
  return &THPVariable_Unpack(o);
}
int64_t number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused("");
  return v;
}
int32_t number32(PyObject* o, const char* what) {
  const int64_t v = number(o);
  require(v >= INT32_MIN && v <= INT32_MAX, what);
  return (int32_t)v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused("");
  return v;
}
// (a tensor without elements has no address, which the library takes for an
// argument that was not given: where that is not the same, the sizes are checked first)
void* address(const at::Tensor* t) { return t ? const_cast<void*>(t->const_data_ptr()) : nullptr; }

bool has_shape(const at::Tensor& t, std::initializer_list<int64_t> shape) {
  return t.sizes().equals(c10::IntArrayRef(shape));
}
// contiguous, of this type and shape (None: fine)
void check(const at::Tensor* t, at::ScalarType type, std::initializer_list<int64_t> shape, const char* what) {
  require(!t || (t->scalar_type() == type && has_shape(*t, shape) && t->is_contiguous()), what);
}
// a device status word (None: none)
void check_status(const at::Tensor* t) {
  require(!t || (t->scalar_type() == at::kInt && t->numel() > 0), "status: int32, a word at least");
}
// elements between the tokens of t: bf16 [T, heads (0: any), D], a token's heads side by side
int64_t token_stride(const at::Tensor* t, int64_t T, int64_t heads, int64_t D, const char* what) {
  if (t && t->scalar_type() == at::kBFloat16 && t->dim() == 3 && t->size(0) == T && t->size(2) == D &&
      (heads == 0 || t->size(1) == heads) && t->stride(2) == 1 && (t->stride(1) == D || t->size(1) == 1))
    return T > 1 ? t->stride(0) : t->size(1) * D;
  throw Refused(what);
}
void on_gpu(std::initializer_list<const at::Tensor*> all, int device) {
  for (const at::Tensor* t : all)
    require(!t || (t->is_cuda() && t->get_device() == device), "tensors lie on the cache's (the logits') CUDA device");
}

// The raw stream of an integer handle, or the current one for None.  The tensors'
// device has to be the current one, where the library launches (the current stream
// knows it: asked for apart it is 5 % of a small call).
void* stream_of(PyObject* o, int device) {
  const char* other = "the tensors' device is not the current one";
  if (o == Py_None) {
    const c10::cuda::CUDAStream s = c10::cuda::getCurrentCUDAStream();
    require(s.device_index() == device, other);
    return (void*)s.stream();
  }
  void* s = PyLong_AsVoidPtr(o);
  if (!s && PyErr_Occurred()) throw Refused("");
  require(c10::cuda::current_device() == device, other);
  return s;
}
// a PagedCache: the address of its struct (of a PagedCache8: of the larger one that begins
// with it), its device (-1: not a CUDA device)
struct Cache {
  const pced_paged_cache* c;
  int device;
  Cache(PyObject* addr, PyObject* dev)
      : c((const pced_paged_cache*)PyLong_AsVoidPtr(addr)), device((int)number(dev)) {}
  const pced_paged_cache8* eight() const { return (const pced_paged_cache8*)c; }
  void on_gpu() const { require(device >= 0, "the cache's tensors lie on a CUDA device"); }
};

template <typename F>
pced_status without_gil(F f) {
  pced_status st;
  Py_BEGIN_ALLOW_THREADS st = f();
  Py_END_ALLOW_THREADS return st;
}

// (cache, device, q, k, v, rope, tok_start, positions, q_out, status, stream)
template <bool EIGHT>
pced_status kv_append(PyObject* const* a) {
  const Cache cache(a[0], a[1]);
  const pced_paged_cache& c = *cache.c;
  const at::Tensor *q = tensor(a[2], "q"), *k = tensor(a[3], "k"), *v = tensor(a[4], "v"), *rope = tensor(a[5], "rope"),
                   *start = tensor(a[6], "tok_start"), *pos = tensor(a[7], "positions"), *out = tensor(a[8], "q_out"),
                   *status = tensor(a[9], "status");
  require(k && k->dim() == 3, "k: bf16 [T, Hkv, D]");
  const int64_t T = k->size(0);
  const int64_t ks = token_stride(k, T, c.Hkv, c.D, "k: bf16 [T, Hkv, D], a token's heads side by side");
  const int64_t vs = token_stride(v, T, c.Hkv, c.D, "v: bf16 [T, Hkv, D], a token's heads side by side");
  int64_t Hq = c.Hkv, qs = 0;
  if (q) {
    qs = token_stride(q, T, 0, c.D, "q: bf16 [T, Hq, D], a token's heads side by side");
    Hq = q->size(1);
    require(out, "q needs q_out");
    check(out, at::kBFloat16, {T, Hq, c.D}, "q_out: contiguous bf16 [T, Hq, D]");
  } else {
    require(!out, "q_out without q");
  }
  int64_t rows = 0;
  if (rope) {
    require(rope->dim() == 2, "rope: contiguous fp32 [rows, D]");
    rows = rope->size(0);
    check(rope, at::kFloat, {rows, c.D}, "rope: contiguous fp32 [rows, D]");
    require(rows > 0, "rope: a table without rows");
  }
  check(start, at::kInt, {c.S + 1}, "tok_start: int32 [S + 1]");
  check(pos, at::kInt, {T}, "positions: int32 [T]");
  check_status(status);
  require(T <= INT32_MAX && rows <= INT32_MAX, "T, rows: below 2^31");
  cache.on_gpu();
  on_gpu({q, k, v, rope, start, pos, out, status}, cache.device);
  void* s = stream_of(a[10], cache.device);
  return without_gil([&] {
    const auto call = [&](auto f, auto c) {
      return f(c, address(q), qs, address(k), ks, address(v), vs, address(out), (int32_t)Hq,
               (const int32_t*)address(start), (int32_t)T, (const float*)address(rope), (int32_t)rows,
               (const int32_t*)address(pos), (int32_t*)address(status), s);
    };
    return EIGHT ? call(pced_kv_append8, cache.eight()) : call(pced_kv_append, cache.c);
  });
}

// (cache, device, status, stream)
pced_status block_summaries(PyObject* const* a) {
  const Cache cache(a[0], a[1]);
  const at::Tensor* status = tensor(a[2], "status");
  check_status(status);
  cache.on_gpu();
  on_gpu({status}, cache.device);
  void* s = stream_of(a[3], cache.device);
  return without_gil([&] { return pced_block_summaries(cache.c, (int32_t*)address(status), s); });
}

// (cache, device, q, n_sel, n_first, n_last, sel, status, stream)
pced_status block_select(PyObject* const* a) {
  const Cache cache(a[0], a[1]);
  const pced_paged_cache& c = *cache.c;
  const at::Tensor *q = tensor(a[2], "q"), *sel = tensor(a[6], "sel"), *status = tensor(a[7], "status");
  const int32_t n_sel = number32(a[3], "n_sel"), n_first = number32(a[4], "n_first"), n_last = number32(a[5], "n_last");
  const int64_t qs = token_stride(q, c.S, 0, c.D, "q: bf16 [S, Hq, D], a token's heads side by side");
  require(sel, "sel: contiguous int32 [S, Hkv, n_sel]");
  check(sel, at::kInt, {c.S, c.Hkv, n_sel}, "sel: contiguous int32 [S, Hkv, n_sel]");
  check_status(status);
  cache.on_gpu();
  on_gpu({q, sel, status}, cache.device);
  void* s = stream_of(a[8], cache.device);
  return without_gil([&] {
    return pced_block_select(cache.c, address(q), qs, (int32_t)q->size(1), n_sel, n_first, n_last,
                             (int32_t*)address(sel), (int32_t*)address(status), s);
  });
}

// (cache, device, q, sel, total_rows, scale, out, lse, ws, stream)
template <bool EIGHT>
pced_status paged_attention(PyObject* const* a) {
  const Cache cache(a[0], a[1]);
  const pced_paged_cache& c = *cache.c;
  const at::Tensor *q = tensor(a[2], "q"), *sel = tensor(a[3], "sel"), *out = tensor(a[6], "out"),
                   *lse = tensor(a[7], "lse"), *ws = tensor(a[8], "ws");
  const int64_t total_rows = number(a[4]);
  const double scale = real(a[5]);
  const int64_t qs = token_stride(q, c.S, 0, c.D, "q: bf16 [S, Hq, D], a token's heads side by side");
  const int64_t Hq = q->size(1);
  int64_t n_sel = 0;
  if (sel) {
    require(sel->dim() == 3, "sel: contiguous int32 [S, Hkv, n_sel]");
    n_sel = sel->size(2);
    check(sel, at::kInt, {c.S, c.Hkv, n_sel}, "sel: contiguous int32 [S, Hkv, n_sel]");
    require(n_sel > 0, "sel: no place for a block (None: all blocks)");
  }
  require(out && ws, "out, ws: tensors");
  const bool f32 = out->scalar_type() == at::kFloat;
  check(out, f32 ? at::kFloat : at::kBFloat16, {c.S, Hq, c.D}, "out: contiguous fp32 or bf16 [S, Hq, D]");
  check(lse, at::kFloat, {c.S, Hq}, "lse: contiguous fp32 [S, Hq]");
  require(ws->scalar_type() == at::kByte && ws->is_contiguous(), "ws: contiguous uint8 (workspace())");
  require(n_sel <= INT32_MAX, "n_sel: below 2^31");
  cache.on_gpu();
  on_gpu({q, sel, out, lse, ws}, cache.device);
  void* s = stream_of(a[9], cache.device);
  return without_gil([&] {
    const auto call = [&](auto f, auto c) {
      return f(c, address(q), qs, (int32_t)Hq, (const int32_t*)address(sel), (int32_t)n_sel, total_rows, (float)scale,
               address(out), f32 ? PCED_OUT_F32 : PCED_OUT_BF16, (float*)address(lse), address(ws),
               (size_t)ws->numel(), s);
    };
    return EIGHT ? call(pced_paged_attention8, cache.eight()) : call(pced_paged_attention, cache.c);
  });
}

// (logits, rows_per_query, history, history_len, penalties, bias_ids, bias, mask, mask_row, out, status, stream)
pced_status logits_process(PyObject* const* a) {
  const at::Tensor *x = tensor(a[0], "logits"), *hist = tensor(a[2], "history"), *len = tensor(a[3], "history_len"),
                   *pen = tensor(a[4], "penalties"), *ids = tensor(a[5], "bias_ids"), *bias = tensor(a[6], "bias"),
                   *mask = tensor(a[7], "mask"), *row = tensor(a[8], "mask_row"), *out = tensor(a[9], "out"),
                   *status = tensor(a[10], "status");
  require(x && x->scalar_type() == at::kFloat && x->dim() == 2 && x->stride(1) == 1, "logits: fp32 [rows, V]");
  const int64_t rows = x->size(0), V = x->size(1), R = number(a[1]), stride = rows > 1 ? x->stride(0) : V;
  require(R >= 1 && rows % R == 0, "rows: a multiple of rows_per_query");
  const int64_t B = rows / R;
  require(out && out->scalar_type() == at::kFloat && has_shape(*out, {rows, V}) && out->stride(1) == 1 &&
              (rows == 1 || out->stride(0) == stride),
          "out: fp32 of the shape and stride of logits");
  int64_t n_hist = 0, n_bias = 0, n_masks = 0, words = 0;
  if (hist) {
    require(hist->dim() == 2, "history: contiguous int32 [B, n]");
    n_hist = hist->size(1);
    check(hist, at::kInt, {B, n_hist}, "history: contiguous int32 [B, n]");
    require(len && pen, "history, history_len and penalties go together");
    check(len, at::kInt, {B}, "history_len: int32 [B]");
    check(pen, at::kFloat, {B, 3}, "penalties: fp32 [B, 3]");
    if (n_hist == 0) hist = len = pen = nullptr;
  } else {
    require(!len && !pen, "history_len and penalties need a history");
  }
  if (ids) {
    require(ids->dim() == 2 && bias, "bias_ids: contiguous int32 [B, n], with bias");
    n_bias = ids->size(1);
    check(ids, at::kInt, {B, n_bias}, "bias_ids: contiguous int32 [B, n]");
    check(bias, at::kFloat, {B, n_bias}, "bias: contiguous fp32 [B, n]");
    if (n_bias == 0) ids = bias = nullptr;
  } else {
    require(!bias, "bias needs bias_ids");
  }
  if (mask) {
    require(mask->dim() == 2, "mask: contiguous int32 [n_masks, words]");
    n_masks = mask->size(0), words = mask->size(1);
    check(mask, at::kInt, {n_masks, words}, "mask: contiguous int32 [n_masks, words]");
    require(n_masks > 0 && words > 0, "mask: no masks, or masks without words");
    check(row, at::kInt, {B}, "mask_row: int32 [B]");
  } else {
    require(!row, "mask_row needs a mask");
  }
  check_status(status);
  for (const int64_t n : {B, R, V, n_hist, n_bias, n_masks, words}) require(n <= INT32_MAX, "sizes: below 2^31");
  require(x->is_cuda(), "logits: on a CUDA device");
  on_gpu({x, hist, len, pen, ids, bias, mask, row, out, status}, x->get_device());
  void* s = stream_of(a[11], x->get_device());
  return without_gil([&] {
    return pced_logits_process((const float*)address(x), (float*)address(out), stride, (int32_t)B, (int32_t)R,
                               (int32_t)V, (const int32_t*)address(hist), (int32_t)n_hist,
                               (const int32_t*)address(len), (const float*)address(pen), (const int32_t*)address(ids),
                               (const float*)address(bias), (int32_t)n_bias, (const uint32_t*)address(mask),
                               (int32_t)n_masks, (int32_t)words, (const int32_t*)address(row),
                               (int32_t*)address(status), s);
  });
}

// (logits, u, temperature, top_k, top_p, min_p, token, logprob, status, stream)
pced_status sample(PyObject* const* a) {
  const at::Tensor *x = tensor(a[0], "logits"), *u = tensor(a[1], "u"), *t = tensor(a[2], "temperature"),
                   *k = tensor(a[3], "top_k"), *p = tensor(a[4], "top_p"), *low = tensor(a[5], "min_p"),
                   *token = tensor(a[6], "token"), *logprob = tensor(a[7], "logprob"), *status = tensor(a[8], "status");
  require(x && (x->scalar_type() == at::kFloat || x->scalar_type() == at::kBFloat16) && x->dim() == 2 &&
              (x->stride(1) == 1 || x->size(1) == 1),
          "logits: fp32 or bf16 [rows, V]");
  const int64_t rows = x->size(0), V = x->size(1), stride = rows > 1 ? x->stride(0) : V;
  require(V > 0, "logits: no tokens");
  require(u && token, "u, token: tensors");
  check(u, at::kFloat, {rows}, "u: fp32 [rows]");
  check(t, at::kFloat, {rows}, "temperature: fp32 [rows]");
  check(k, at::kInt, {rows}, "top_k: int32 [rows]");
  check(p, at::kFloat, {rows}, "top_p: fp32 [rows]");
  check(low, at::kFloat, {rows}, "min_p: fp32 [rows]");
  check(token, at::kInt, {rows}, "token: int32 [rows]");
  check(logprob, at::kFloat, {rows}, "logprob: fp32 [rows]");
  check_status(status);
  require(rows <= INT32_MAX && V <= INT32_MAX, "sizes: below 2^31");
  require(x->is_cuda(), "logits: on a CUDA device");
  on_gpu({x, u, t, k, p, low, token, logprob, status}, x->get_device());
  void* s = stream_of(a[9], x->get_device());
  return without_gil([&] {
    return pced_sample(address(x), x->scalar_type() == at::kFloat ? PCED_IN_F32 : PCED_IN_BF16, stride, (int32_t)rows,
                       (int32_t)V, (const float*)address(u), (const float*)address(t), (const int32_t*)address(k),
                       (const float*)address(p), (const float*)address(low), (int32_t*)address(token),
                       (float*)address(logprob), (int32_t*)address(status), s);
  });
}

// A call's status as a Python number; no C++ exception leaves it.
template <pced_status (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments", N);
    return nullptr;
  }
  try {
    return PyLong_FromLong(F(args));
  } catch (const Refused& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

template <pced_status (*F)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
  return {name, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<kv_append<false>, 11>("kv_append"),
                         method<kv_append<true>, 11>("kv_append8"),
                         method<block_summaries, 4>("block_summaries"),
                         method<block_select, 9>("block_select"),
                         method<paged_attention<false>, 10>("paged_attention"),
                         method<paged_attention<true>, 10>("paged_attention8"),
                         method<logits_process, 12>("logits_process"),
                         method<sample, 10>("sample"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "pced_calls", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_pced_calls(void) { return PyModule_Create(&module); }
