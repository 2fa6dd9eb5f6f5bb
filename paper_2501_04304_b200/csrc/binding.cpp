// Native half of binding.py: the hot-path calls of libdgq with their output and workspace allocations, as
// positional CPython functions.  A layer pass is two library calls, five allocations and two or three kernel
// launches; marshalling them through ctypes and torch.empty took 38 us of host time (256 x 320 x 320, static
// tables), more than the kernels of every small layer.  Keyword handling, defaults and the meaning of
// every argument live in binding.py.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/dgq.h"

namespace {

at::Tensor empty(std::initializer_list<int64_t> shape, at::ScalarType type, const at::Tensor& like) {
  return at::Tensor(at::detail::empty_cuda(at::IntArrayRef(shape.begin(), shape.size()), type, like.device(), std::nullopt));
}

// Scratch memory for a call on stream `st` that is dropped when the call returns: it belongs to that stream, so that torch
// gives it to nobody else before the call's kernels have run.  `given` is the stream argument (None: the current
// stream, to which torch's allocations belong anyway).
at::Tensor scratch(int64_t bytes, const at::Tensor& like, PyObject* given, void* st) {
  if (given == Py_None) return empty({bytes}, at::kByte, like);
  c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), like.device().index()));
  return empty({bytes}, at::kByte, like);
}

// A tensor argument, or an undefined tensor for None.  Sets a TypeError for anything else.
bool tensor(PyObject* o, at::Tensor* t) {
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor or None, got %s", Py_TYPE(o)->tp_name);
    return false;
  }
  *t = THPVariable_Unpack(o);
  return true;
}

template <typename T = void>
T* ptr(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

PyObject* wrap(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}

// An integer argument; one that 32 bits do not hold is refused, not cut.
bool integer(PyObject* o, int* v) {
  const long x = PyLong_AsLong(o);
  if (x == -1 && PyErr_Occurred()) return false;
  if (x < INT32_MIN || x > INT32_MAX) {
    PyErr_SetString(PyExc_ValueError, "an integer argument does not fit 32 bits");
    return false;
  }
  *v = static_cast<int>(x);
  return true;
}

// The argument of a stream parameter: None (the current stream) or an object with a `cuda_stream` handle.
bool stream_arg(PyObject* o, void** s) {
  if (o == Py_None) {
    *s = c10::cuda::getCurrentCUDAStream().stream();
    return true;
  }
  static PyObject* name = PyUnicode_InternFromString("cuda_stream");
  PyObject* v = PyObject_GetAttr(o, name);
  if (!v) return false;
  *s = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

bool handle(PyObject* o, void** h) {
  *h = PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}

// binding.py raises DgqError from a status returned in place of a result.
PyObject* status(dgq_status st) { return PyLong_FromLong(st); }

// A function of the module: what torch's C++ API throws (no CUDA device, a tensor without storage, a dimension that
// is not there) becomes a Python exception.  For that everything that may throw, taking a tensor's address included,
// runs with the GIL held: between Py_BEGIN_ALLOW_THREADS and its end stands nothing but the library call.
template <PyObject* (*BODY)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return BODY(a, n);
  } catch (python_error& e) {
    e.restore();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// A tuple of the objects, whose references it takes over; null if one of them is.
PyObject* tuple(std::initializer_list<PyObject*> items) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(items.size()));
  bool ok = r != nullptr;
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    ok = ok && o;
    if (r) PyTuple_SET_ITEM(r, i++, o);
    else Py_XDECREF(o);
  }
  if (!ok) Py_CLEAR(r);
  return r;
}

// An output: the caller's buffer as the object it is, or the tensor made for it.
PyObject* output(PyObject* given, const at::Tensor& t) { return given == Py_None ? wrap(t) : Py_NewRef(given); }

bool require(bool ok, const char* what) {
  if (!ok) PyErr_SetString(PyExc_AssertionError, what);
  return ok;
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

// (groups, K_pad, G, timestep, mode, layout, X, out | None, scale | None, zp | None, allocate, stream) -> (Xq, scale, zp)
PyObject* quantize_act(PyObject* const* a, Py_ssize_t n) {
  void *g, *st;
  int k_pad, n_groups, timestep, mode, layout, allocate;
  at::Tensor x, out, scale, zp;
  if (!arity(n, 12) || !handle(a[0], &g) || !integer(a[1], &k_pad) || !integer(a[2], &n_groups) ||
      !integer(a[3], &timestep) || !integer(a[4], &mode) || !integer(a[5], &layout) || !tensor(a[6], &x) ||
      !tensor(a[7], &out) || !tensor(a[8], &scale) || !tensor(a[9], &zp) || !integer(a[10], &allocate) ||
      !stream_arg(a[11], &st))
    return nullptr;
  if (!require(x.defined() && x.is_cuda() && x.scalar_type() == at::kHalf && x.dim() == 2 && x.stride(1) == 1,
               "X is a CUDA fp16 matrix with contiguous rows"))
    return nullptr;
  const int64_t m = x.size(0);
  if (allocate) {
    if (!out.defined()) out = empty({m, k_pad}, at::kByte, x);
    if (mode == DGQ_MODE_DYNAMIC_TOKEN) {
      scale = empty({m, n_groups}, at::kFloat, x);
      zp = empty({m, n_groups}, at::kInt, x);
    }
  }
  const int64_t ld = x.stride(0);
  void *p_x = ptr(x), *p_out = ptr(out);
  float* p_scale = ptr<float>(scale);
  int32_t* p_zp = ptr<int32_t>(zp);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_quantize_act(static_cast<const dgq_groups*>(g), timestep, mode, layout, p_x, m, ld, p_out, p_scale, p_zp, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return tuple({output(a[7], out), wrap(scale), wrap(zp)});
}

// (groups, weight, N, timestep, mode, layout, Xq, scale, zp, bias, out | None, conv | None, workspace, stream) -> Y
// workspace: a tensor, None (one of the size the library asks for) or False (none).
PyObject* linear(PyObject* const* a, Py_ssize_t n) {
  void *g, *w, *st;
  int n_out, timestep, mode, layout;
  at::Tensor xq, scale, zp, bias, y, ws;
  if (!arity(n, 14) || !handle(a[0], &g) || !handle(a[1], &w) || !integer(a[2], &n_out) || !integer(a[3], &timestep) ||
      !integer(a[4], &mode) || !integer(a[5], &layout) || !tensor(a[6], &xq) || !tensor(a[7], &scale) ||
      !tensor(a[8], &zp) || !tensor(a[9], &bias) || !tensor(a[10], &y) ||
      (a[12] != Py_False && !tensor(a[12], &ws)) || !stream_arg(a[13], &st))
    return nullptr;
  dgq_conv_desc conv;
  if (a[11] != Py_None) {
    PyObject* t = PySequence_Tuple(a[11]);
    if (!t) return nullptr;
    const bool ok = PyArg_ParseTuple(t, "iiii", &conv.n, &conv.h, &conv.w, &conv.c);
    Py_DECREF(t);
    if (!ok) return nullptr;
  }
  if (!require(xq.defined() && xq.dim() >= 1, "Xq is a matrix of codes")) return nullptr;
  const int64_t m = xq.size(0);
  if (!y.defined()) y = empty({m, n_out}, at::kHalf, xq);
  dgq_status rc = DGQ_OK;
  if (a[12] == Py_None) {
    size_t need = 0;
    rc = dgq_linear_workspace_bytes(static_cast<const dgq_groups*>(g), static_cast<const dgq_weight*>(w), m, &need);
    if (rc != DGQ_OK) return status(rc);
    if (need) ws = scratch(static_cast<int64_t>(need), xq, a[13], st);
  }
  const int64_t ldy = y.stride(0);
  const size_t ws_bytes = ws.defined() ? static_cast<size_t>(ws.numel()) : 0;
  void *p_xq = ptr(xq), *p_bias = ptr(bias), *p_y = ptr(y), *p_ws = ptr(ws);
  float* p_scale = ptr<float>(scale);
  int32_t* p_zp = ptr<int32_t>(zp);
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_linear(static_cast<const dgq_groups*>(g), static_cast<const dgq_weight*>(w), timestep, mode, layout, p_xq, p_scale,
                  p_zp, p_bias, p_y, m, ldy, a[11] != Py_None ? &conv : nullptr, p_ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return output(a[10], y);
}

// (Q, K, V, score_bits, scale_gran, fixed_scale, out | None, want_scale, want_codes, workspace | None, v_bits, stream)
// -> (O, scale, codes)
PyObject* cross_attn_logq(PyObject* const* a, Py_ssize_t n) {
  void* st;
  int bits, gran, want_scale, want_codes, v_bits;
  at::Tensor q, k, v, fixed, o, scale, codes, ws;
  if (!arity(n, 12) || !tensor(a[0], &q) || !tensor(a[1], &k) || !tensor(a[2], &v) || !integer(a[3], &bits) ||
      !integer(a[4], &gran) || !tensor(a[5], &fixed) || !tensor(a[6], &o) || !integer(a[7], &want_scale) ||
      !integer(a[8], &want_codes) || !tensor(a[9], &ws) || !integer(a[10], &v_bits) || !stream_arg(a[11], &st))
    return nullptr;
  if (!require(q.defined() && k.defined() && v.defined() && q.dim() == 4 && q.is_contiguous() && k.is_contiguous() &&
                   v.is_contiguous(),
               "Q, K and V are contiguous [B, n, H, d] tensors"))
    return nullptr;
  const int64_t B = q.size(0), nq = q.size(1), H = q.size(2), d = q.size(3), nk = k.size(1);
  if (!o.defined()) o = empty({B, nq, H, d}, q.scalar_type(), q);
  if (want_scale) {
    const int64_t scopes = gran == DGQ_SCALE_PER_PROMPT ? B : gran == DGQ_SCALE_PER_PROMPT_HEAD ? B * H : 1;
    scale = empty({scopes}, at::kFloat, q);
  }
  if (want_codes) codes = empty({B, H, nq, nk - 1}, at::kByte, q);
  if (!ws.defined()) {
    size_t need = 256;
    if (nk >= 2) {
      const dgq_status rc = dgq_cross_attn_workspace_bytes(B, H, nq, nk, d, &need);
      if (rc != DGQ_OK) return status(rc);
    }
    ws = scratch(static_cast<int64_t>(need), q, a[11], st);
  }
  void *p_q = ptr(q), *p_k = ptr(k), *p_v = ptr(v), *p_o = ptr(o), *p_ws = ptr(ws);
  float *p_fixed = ptr<float>(fixed), *p_scale = ptr<float>(scale);
  uint8_t* p_codes = ptr<uint8_t>(codes);
  const size_t ws_bytes = ws.numel();
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  if (v_bits)
    rc = dgq_cross_attn_logq_qv(p_q, p_k, p_v, B, H, nq, nk, d, bits, gran, p_fixed, v_bits, p_o, p_scale, p_codes, p_ws, ws_bytes, st);
  else
    rc = dgq_cross_attn_logq(p_q, p_k, p_v, B, H, nq, nk, d, bits, gran, p_fixed, p_o, p_scale, p_codes, p_ws, ws_bytes, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return tuple({output(a[6], o), wrap(scale), wrap(codes)});
}

// (Q, K, V, score_bits, fixed_scale, out | None, want_codes, stream) -> (O, codes)
PyObject* self_attn_logq(PyObject* const* a, Py_ssize_t n) {
  void* st;
  int bits, want_codes;
  at::Tensor q, k, v, fixed, o, codes;
  if (!arity(n, 8) || !tensor(a[0], &q) || !tensor(a[1], &k) || !tensor(a[2], &v) || !integer(a[3], &bits) ||
      !tensor(a[4], &fixed) || !tensor(a[5], &o) || !integer(a[6], &want_codes) || !stream_arg(a[7], &st))
    return nullptr;
  if (!require(q.defined() && k.defined() && v.defined() && q.dim() == 4 && q.is_contiguous() && k.is_contiguous() &&
                   v.is_contiguous(),
               "Q, K and V are contiguous [B, n, H, d] tensors"))
    return nullptr;
  const int64_t B = q.size(0), nq = q.size(1), H = q.size(2), d = q.size(3), nk = k.size(1);
  if (!o.defined()) o = empty({B, nq, H, d}, q.scalar_type(), q);
  if (want_codes) codes = empty({B, H, nq, nk}, at::kByte, q);
  void *p_q = ptr(q), *p_k = ptr(k), *p_v = ptr(v), *p_o = ptr(o);
  float* p_fixed = ptr<float>(fixed);
  uint8_t* p_codes = ptr<uint8_t>(codes);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_self_attn_logq(p_q, p_k, p_v, B, H, nq, nk, d, bits, p_fixed, p_o, p_codes, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return tuple({output(a[5], o), wrap(codes)});
}

// ---------------------------------------------------------------- attention over encoder states and over the 8-bit cache
// These calls go to the device of their first tensor, whichever is current, and check shapes before the library sees a pointer.

bool fail(const char* what) {
  PyErr_SetString(PyExc_ValueError, what);
  return false;
}

// Type, device, innermost stride and (for its two or three outer dimensions) the strides of a 16-bit tensor.
bool rows16(const at::Tensor& t, const at::Tensor& like, int64_t dims, const char* what, dgq_rows* r) {
  if (!t.defined() || !t.is_cuda() || t.device() != like.device() || t.scalar_type() != like.scalar_type() || t.dim() != dims ||
      (t.scalar_type() != at::kHalf && t.scalar_type() != at::kBFloat16) || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1))
    return fail(what);
  *r = dgq_rows{t.data_ptr(), dims == 4 ? t.stride(0) : 0, t.stride(dims - 3), t.stride(dims - 2)};
  return true;
}

bool ints(const at::Tensor& t, const at::Tensor& like, const char* what) {
  if (!t.is_cuda() || t.device() != like.device() || t.scalar_type() != at::kInt || !t.is_contiguous()) return fail(what);
  return true;
}

bool fits(int64_t v, int* out) {
  if (v > INT32_MAX) return fail("a size is beyond 2^31");
  *out = static_cast<int>(v);
  return true;
}

int dtype_of(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? DGQ_BF16 : DGQ_F16; }

// The stream for a call on `like`'s device: the given one or that device's current one.
bool stream_on(PyObject* o, const at::Tensor& like, void** st) {
  if (o == Py_None) {
    *st = c10::cuda::getCurrentCUDAStream(like.device().index()).stream();
    return true;
  }
  return stream_arg(o, st);
}

// An output made here that a stream other than the current one writes: torch gives its memory to nobody else before that has
// happened, even if the caller drops it.
void on_stream(const at::Tensor& t, PyObject* given, void* st) {
  if (given != Py_None)
    c10::cuda::CUDACachingAllocator::recordStream(
        t.storage().data_ptr(), c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), t.device().index()));
}

// n elements of a one-dimensional tensor as a tensor of their own (in the same storage).
at::Tensor part(const at::Tensor& all, int64_t first, int64_t n) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
  t.unsafeGetTensorImpl()->set_sizes_contiguous(at::IntArrayRef(&n, 1));
  t.unsafeGetTensorImpl()->set_storage_offset(first);
  return t;
}

bool scale_arg(PyObject* o, int64_t d, float* scale) {
  if (o == Py_None) {
    *scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(d)));
    return true;
  }
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) return false;
  *scale = static_cast<float>(v);
  return true;
}

// (k, v, k_scale, v_scale, d): codes [pages, heads, page, row], scales [pages, heads]
bool cache_arg(PyObject* const* a, at::Tensor* k, dgq_kv_cache* c) {
  at::Tensor v, ks, vs;
  if (!tensor(a[0], k) || !tensor(a[1], &v) || !tensor(a[2], &ks) || !tensor(a[3], &vs) || !integer(a[4], &c->d)) return false;
  if (!k->defined() || !v.defined() || !ks.defined() || !vs.defined() || !k->is_cuda() || k->dim() != 4 || v.sizes() != k->sizes() ||
      ks.dim() != 2 || ks.size(0) != k->size(0) || ks.size(1) != k->size(1) || vs.sizes() != ks.sizes() ||
      k->scalar_type() != at::kChar || v.scalar_type() != at::kChar || ks.scalar_type() != at::kFloat ||
      vs.scalar_type() != at::kFloat || !k->is_contiguous() || !v.is_contiguous() || !ks.is_contiguous() || !vs.is_contiguous() ||
      v.device() != k->device() || ks.device() != k->device() || vs.device() != k->device())
    return fail("a cache is contiguous CUDA int8 codes [pages, heads, page, row] and fp32 scales [pages, heads]");
  if (c->d <= 0 || k->size(3) != (c->d + 15) / 16 * 16) return fail("a cache's rows are d codes rounded up to a multiple of 16");
  int page;
  if (!fits(k->size(0), &c->n_pages) || !fits(k->size(1), &c->n_heads) || !fits(k->size(2), &page)) return false;
  c->page = page;
  c->k = k->data_ptr();
  c->v = v.data_ptr();
  c->k_scale = static_cast<float*>(ks.data_ptr());
  c->v_scale = static_cast<float*>(vs.data_ptr());
  return true;
}

// (Q, K, V, kv_lens | None, scale | None, out | None, stream) -> O
PyObject* encoder_attn(PyObject* const* a, Py_ssize_t n) {
  void* st;
  at::Tensor q, k, v, lens, o;
  dgq_rows rq, rk, rv, ro;
  float scale;
  if (!arity(n, 7) || !tensor(a[0], &q) || !tensor(a[1], &k) || !tensor(a[2], &v) || !tensor(a[3], &lens) || !tensor(a[5], &o)) return nullptr;
  if (!rows16(q, q, 4, "Q is a CUDA fp16 or bf16 tensor [B, nq, Hq, d] with contiguous rows", &rq) ||
      !rows16(k, q, 4, "K is a tensor [B, nk, Hkv, d] of Q's type and device with contiguous rows", &rk) ||
      !rows16(v, q, 4, "V is a tensor [B, nk, Hkv, d] of Q's type and device with contiguous rows", &rv))
    return nullptr;
  int B, nq, hq, d, nk, hkv;
  if (!fits(q.size(0), &B) || !fits(q.size(1), &nq) || !fits(q.size(2), &hq) || !fits(q.size(3), &d) || !fits(k.size(1), &nk) ||
      !fits(k.size(2), &hkv))
    return nullptr;
  if ((k.size(0) != B || k.size(3) != d || v.sizes() != k.sizes()) && !fail("K and V are [B, nk, Hkv, d] with Q's B and d")) return nullptr;
  if (lens.defined() && (!ints(lens, q, "kv_lens is a contiguous CUDA int32 tensor [B]") ||
                         (lens.numel() != B && !fail("kv_lens has one length a request"))))
    return nullptr;
  if (!scale_arg(a[4], d, &scale)) return nullptr;
  const c10::cuda::CUDAGuard on(q.device());
  if (!stream_on(a[6], q, &st)) return nullptr;
  if (!o.defined()) {
    o = empty({B, nq, hq, d}, q.scalar_type(), q);
    on_stream(o, a[6], st);
  }
  if (!rows16(o, q, 4, "out is a tensor like Q", &ro) || (o.sizes() != q.sizes() && !fail("out is a tensor like Q"))) return nullptr;
  if (o.numel() == 0) return output(a[5], o);
  if (nk == 0) {
    if (st == c10::cuda::getCurrentCUDAStream().stream()) {
      o.zero_();
    } else {
      c10::cuda::CUDAStreamGuard there(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), q.device().index()));
      o.zero_();
    }
    return output(a[5], o);
  }
  const int32_t* p_lens = ptr<int32_t>(lens);
  const int type = dtype_of(q);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_encoder_attn(&rq, &rk, &rv, &ro, type, B, hq, hkv, nq, nk, d, scale, p_lens, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return output(a[5], o);
}

// (k, v, k_scale, v_scale, d, Q, block_table, kv_lens, q_start | None, max_nq | None, causal, scale | None, out | None, stream) -> O
PyObject* cached_attn(PyObject* const* a, Py_ssize_t n) {
  void* st;
  dgq_kv_cache c;
  at::Tensor kc, q, table, lens, start, o;
  dgq_rows rq, ro;
  float scale;
  int causal, max_nq, B, hq, max_pages;
  if (!arity(n, 14) || !cache_arg(a, &kc, &c) || !tensor(a[5], &q) || !tensor(a[6], &table) || !tensor(a[7], &lens) ||
      !tensor(a[8], &start) || !integer(a[10], &causal) || !tensor(a[12], &o))
    return nullptr;
  const int dims = start.defined() ? 3 : 4;
  if (!rows16(q, q, dims, "Q is a CUDA fp16 or bf16 tensor [B, nq, Hq, d] or, with q_start, [rows, Hq, d]; rows contiguous", &rq)) return nullptr;
  if ((q.device() != kc.device() || q.size(dims - 1) != c.d) && !fail("Q has the cache's d and device")) return nullptr;
  if ((!table.defined() || !lens.defined() || table.dim() != 2 || lens.dim() != 1 || lens.size(0) != table.size(0)) &&
      !fail("block_table is [B, max_pages], kv_lens [B]"))
    return nullptr;
  if (!ints(table, q, "block_table is a contiguous CUDA int32 tensor") || !ints(lens, q, "kv_lens is a contiguous CUDA int32 tensor")) return nullptr;
  if (!fits(table.size(0), &B) || !fits(table.size(1), &max_pages) || !fits(q.size(dims - 2), &hq)) return nullptr;
  if (start.defined()) {
    if (!ints(start, q, "q_start is a contiguous CUDA int32 tensor [B + 1]") || (start.numel() != B + 1ll && !fail("q_start is [B + 1]"))) return nullptr;
    if (a[9] == Py_None) {
      if (!fits(q.size(0), &max_nq)) return nullptr;
    } else if (!integer(a[9], &max_nq)) {
      return nullptr;
    }
  } else {
    if (!fits(q.size(1), &max_nq) || (q.size(0) != B && !fail("Q has one entry a request"))) return nullptr;
    if (a[9] != Py_None) {
      int given;
      if (!integer(a[9], &given) || (given != max_nq && !fail("max_nq is Q's own where there is no q_start"))) return nullptr;
    }
  }
  if (!scale_arg(a[11], c.d, &scale)) return nullptr;
  const c10::cuda::CUDAGuard on(q.device());
  if (!stream_on(a[13], q, &st)) return nullptr;
  if (!o.defined()) {
    o = dims == 4 ? empty({B, max_nq, hq, c.d}, q.scalar_type(), q) : empty({q.size(0), hq, c.d}, q.scalar_type(), q);
    on_stream(o, a[13], st);
  }
  if (!rows16(o, q, dims, "out is a tensor like Q", &ro) || (o.sizes() != q.sizes() && !fail("out is a tensor like Q"))) return nullptr;
  if (o.numel() == 0 || B == 0) return output(a[12], o);
  const int64_t n_rows = q.size(0);
  const int32_t *p_table = ptr<int32_t>(table), *p_lens = ptr<int32_t>(lens), *p_start = ptr<int32_t>(start);
  const int type = dtype_of(q);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_cached_attn(&c, &rq, &ro, type, B, hq, n_rows, p_start, max_nq, p_table, max_pages, p_lens, causal, scale, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return output(a[12], o);
}

// (k, v, k_scale, v_scale, d, K, V, slots, stream) -> None
PyObject* kv_write(PyObject* const* a, Py_ssize_t n) {
  void* st;
  dgq_kv_cache c;
  at::Tensor kc, k, v, slots;
  dgq_rows rk, rv;
  if (!arity(n, 9) || !cache_arg(a, &kc, &c) || !tensor(a[5], &k) || !tensor(a[6], &v) || !tensor(a[7], &slots)) return nullptr;
  if (!rows16(k, k, 3, "K is a CUDA fp16 or bf16 tensor [T, heads, d] with contiguous rows", &rk) ||
      !rows16(v, k, 3, "V is a tensor [T, heads, d] of K's type and device with contiguous rows", &rv))
    return nullptr;
  if ((k.device() != kc.device() || v.sizes() != k.sizes() || k.size(1) != c.n_heads || k.size(2) != c.d || !slots.defined() ||
       slots.numel() != k.size(0)) &&
      !fail("K and V are [T, heads, d] of the cache's heads, d and device, slots [T]"))
    return nullptr;
  if (!ints(slots, k, "slots is a contiguous CUDA int32 tensor [T]")) return nullptr;
  const int64_t T = k.size(0);
  if (T == 0) Py_RETURN_NONE;
  const c10::cuda::CUDAGuard on(k.device());
  if (!stream_on(a[8], k, &st)) return nullptr;
  const int32_t* p_slots = ptr<int32_t>(slots);
  const int type = dtype_of(k);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_kv_write(&c, &rk, &rv, type, T, p_slots, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  Py_RETURN_NONE;
}

// (k, v, k_scale, v_scale, d, slots, bf16, K | None, V | None, stream) -> (K, V)
PyObject* kv_read(PyObject* const* a, Py_ssize_t n) {
  void* st;
  dgq_kv_cache c;
  at::Tensor kc, slots, out[2];
  dgq_rows r[2];
  int bf16;
  if (!arity(n, 10) || !cache_arg(a, &kc, &c) || !tensor(a[5], &slots) || !integer(a[6], &bf16) || !tensor(a[7], &out[0]) ||
      !tensor(a[8], &out[1]))
    return nullptr;
  if (!slots.defined() && !fail("slots is a contiguous CUDA int32 tensor [T]")) return nullptr;
  if (!ints(slots, kc, "slots is a contiguous CUDA int32 tensor [T]")) return nullptr;
  const int64_t T = slots.numel();
  const at::ScalarType want = bf16 ? at::kBFloat16 : at::kHalf;
  const c10::cuda::CUDAGuard on(kc.device());
  if (!stream_on(a[9], kc, &st)) return nullptr;
  for (int i = 0; i < 2; ++i) {
    if (!out[i].defined()) {
      out[i] = empty({T, c.n_heads, c.d}, want, kc);
      on_stream(out[i], a[9], st);
    }
    if (!rows16(out[i], out[i], 3, "outputs are [T, heads, d] with contiguous rows", &r[i])) return nullptr;
    if ((out[i].scalar_type() != want || out[i].device() != kc.device() || out[i].size(0) != T || out[i].size(1) != c.n_heads ||
         out[i].size(2) != c.d) &&
        !fail("outputs are [T, heads, d] of the asked type on the cache's device"))
      return nullptr;
  }
  if (T > 0) {
    const int32_t* p_slots = ptr<int32_t>(slots);
    dgq_status rc;
    Py_BEGIN_ALLOW_THREADS
    rc = dgq_kv_read(&c, p_slots, T, &r[0], &r[1], bf16 ? DGQ_BF16 : DGQ_F16, st);
    Py_END_ALLOW_THREADS
    if (rc != DGQ_OK) return status(rc);
  }
  return tuple({output(a[7], out[0]), output(a[8], out[1])});
}

// (lens, n_new, free_pages, block_table, page, n_tokens, stream) -> (token_start, kv_lens, slots, used)
PyObject* kv_plan(PyObject* const* a, Py_ssize_t n) {
  void* st;
  at::Tensor lens, add, pages, table;
  int page, n_tokens, B, max_pages, n_free;
  if (!arity(n, 7) || !tensor(a[0], &lens) || !tensor(a[1], &add) || !tensor(a[2], &pages) || !tensor(a[3], &table) ||
      !integer(a[4], &page) || !integer(a[5], &n_tokens))
    return nullptr;
  if ((!lens.defined() || !add.defined() || !pages.defined() || !table.defined() || table.dim() != 2 || lens.dim() != 1 ||
       add.dim() != 1 || lens.size(0) != table.size(0) || add.size(0) != table.size(0) || n_tokens < 0) &&
      !fail("lens and n_new are [B], block_table [B, max_pages], n_tokens is not negative"))
    return nullptr;
  if (!ints(lens, lens, "lens is a contiguous CUDA int32 tensor") || !ints(add, lens, "n_new is a contiguous CUDA int32 tensor") ||
      !ints(pages, lens, "free_pages is a contiguous CUDA int32 tensor") || !ints(table, lens, "block_table is a contiguous CUDA int32 tensor"))
    return nullptr;
  if (!fits(table.size(0), &B) || !fits(table.size(1), &max_pages) || !fits(pages.numel(), &n_free)) return nullptr;
  const c10::cuda::CUDAGuard on(lens.device());
  if (!stream_on(a[6], lens, &st)) return nullptr;
  // one allocation for the four outputs (three more cost the call 1.4 us of 6.3)
  const at::Tensor all = empty({2ll * B + 2 + n_tokens}, at::kInt, lens);
  on_stream(all, a[6], st);
  at::Tensor start = part(all, 0, B + 1ll), out_lens = part(all, B + 1ll, B), slots = part(all, 2ll * B + 1, n_tokens),
             used = part(all, 2ll * B + 1 + n_tokens, 1);
  const int32_t *p_lens = ptr<int32_t>(lens), *p_add = ptr<int32_t>(add), *p_pages = ptr<int32_t>(pages);
  int32_t *p_table = ptr<int32_t>(table), *p_start = ptr<int32_t>(start), *p_out = ptr<int32_t>(out_lens), *p_slots = ptr<int32_t>(slots),
          *p_used = ptr<int32_t>(used);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_kv_plan(p_lens, p_add, B, p_pages, n_free, p_table, max_pages, page, p_start, p_out, p_slots, n_tokens, p_used, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return tuple({wrap(start), wrap(out_lens), wrap(slots), wrap(used)});
}

// ---------------------------------------------------------------- group norm and products of few rows
bool floats(const at::Tensor& t, const at::Tensor& like, int64_t n, const char* what) {
  if (t.defined() && (!t.is_cuda() || t.device() != like.device() || t.scalar_type() != at::kFloat || !t.is_contiguous() || t.numel() != n))
    return fail(what);
  return true;
}

// A map [B, P, C] or [B, H, W, C] whose pixels lie at one distance from each other.
bool map16(const at::Tensor& t, const at::Tensor& like, const char* what, dgq_rows* r, int64_t* pixels) {
  const int64_t dims = t.defined() ? t.dim() : 0;
  if (!t.defined() || !t.is_cuda() || t.device() != like.device() || t.scalar_type() != like.scalar_type() || (dims != 3 && dims != 4) ||
      (t.scalar_type() != at::kHalf && t.scalar_type() != at::kBFloat16) || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1))
    return fail(what);
  int64_t step = t.stride(dims - 2);
  *pixels = t.size(1);
  if (dims == 4) {
    *pixels *= t.size(2);
    if (t.size(2) == 1) step = t.stride(1);
    else if (t.size(1) > 1 && t.stride(1) != t.size(2) * step) return fail(what);
  }
  *r = dgq_rows{t.data_ptr(), t.stride(0), step, 0};
  return true;
}

struct NormArgs {
  at::Tensor x, gamma, beta, add;
  dgq_rows rx;
  int B, P, C, n_groups, act;
  float eps;
  int64_t ld_add;
};
// (X, n_groups, gamma | None, beta | None, eps, act, add | None)
bool norm_args(PyObject* const* a, NormArgs* n) {
  if (!tensor(a[0], &n->x) || !integer(a[1], &n->n_groups) || !tensor(a[2], &n->gamma) || !tensor(a[3], &n->beta) || !integer(a[5], &n->act) ||
      !tensor(a[6], &n->add))
    return false;
  const double eps = PyFloat_AsDouble(a[4]);
  if (eps == -1.0 && PyErr_Occurred()) return false;
  n->eps = static_cast<float>(eps);
  int64_t pixels;
  if (!map16(n->x, n->x, "X is a CUDA fp16 or bf16 map [B, P, C] or [B, H, W, C] with contiguous channels and evenly spaced pixels", &n->rx, &pixels))
    return false;
  if (!fits(n->x.size(0), &n->B) || !fits(pixels, &n->P) || !fits(n->x.size(n->x.dim() - 1), &n->C)) return false;
  if (!floats(n->gamma, n->x, n->C, "gamma is a contiguous CUDA fp32 tensor [C]") || !floats(n->beta, n->x, n->C, "beta is a contiguous CUDA fp32 tensor [C]"))
    return false;
  n->ld_add = 0;
  if (n->add.defined()) {
    if (!n->add.is_cuda() || n->add.device() != n->x.device() || n->add.scalar_type() != n->x.scalar_type() || n->add.dim() != 2 ||
        n->add.size(0) != n->B || n->add.size(1) != n->C || (n->C > 1 && n->add.stride(1) != 1))
      return fail("add is a tensor [B, C] of X's type and device with contiguous rows");
    n->ld_add = n->add.stride(0);
  }
  return true;
}
// The workspace of a call: the caller's, or one of the size the library asks for.
bool norm_workspace(PyObject* given, const NormArgs& n, int quantize, PyObject* stream, void* st, at::Tensor* ws, dgq_status* rc) {
  *rc = DGQ_OK;
  if (!tensor(given, ws)) return false;
  if (ws->defined()) {
    if (!ws->is_cuda() || ws->device() != n.x.device() || !ws->is_contiguous()) return fail("workspace is a contiguous CUDA tensor on X's device");
    return true;
  }
  size_t need = 0;
  *rc = dgq_group_norm_workspace_bytes(n.B, n.P, n.C, n.n_groups, quantize, &need);
  if (*rc == DGQ_OK && need) *ws = scratch(static_cast<int64_t>(need), n.x, stream, st);
  return true;
}

// (X, n_groups, gamma, beta, eps, act, add, out | None, workspace | None, stream) -> Y
PyObject* group_norm(PyObject* const* a, Py_ssize_t n) {
  void* st;
  NormArgs x;
  at::Tensor y, ws;
  if (!arity(n, 10) || !norm_args(a, &x) || !tensor(a[7], &y)) return nullptr;
  const c10::cuda::CUDAGuard on(x.x.device());
  if (!stream_on(a[9], x.x, &st)) return nullptr;
  if (!y.defined()) {
    y = x.x.dim() == 3 ? empty({x.x.size(0), x.x.size(1), x.x.size(2)}, x.x.scalar_type(), x.x)
                       : empty({x.x.size(0), x.x.size(1), x.x.size(2), x.x.size(3)}, x.x.scalar_type(), x.x);
    on_stream(y, a[9], st);
  }
  dgq_rows ry;
  int64_t pixels;
  if (!map16(y, x.x, "out is a map like X", &ry, &pixels) || (y.sizes() != x.x.sizes() && !fail("out is a map like X"))) return nullptr;
  if (y.numel() == 0) return output(a[7], y);
  dgq_status rc;
  if (!norm_workspace(a[8], x, 0, a[9], st, &ws, &rc)) return nullptr;
  if (rc != DGQ_OK) return status(rc);
  const int type = dtype_of(x.x);
  void *p_add = ptr(x.add), *p_ws = ptr(ws);
  const float *p_gamma = ptr<float>(x.gamma), *p_beta = ptr<float>(x.beta);
  const size_t bytes = ws.defined() ? ws.nbytes() : 0;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_group_norm(&x.rx, p_add, x.ld_add, p_gamma, p_beta, &ry, type, x.B, x.P, x.C, x.n_groups, x.eps, x.act, p_ws, bytes, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return output(a[7], y);
}

// (groups, C of the grouping, K_pad, timestep, layout, X, n_groups, gamma, beta, eps, act, add, out | None, workspace | None, stream) -> Xq
PyObject* group_norm_quantize(PyObject* const* a, Py_ssize_t n) {
  void *st, *g;
  int channels, k_pad, timestep, layout;
  NormArgs x;
  at::Tensor xq, ws;
  if (!arity(n, 15) || !handle(a[0], &g) || !integer(a[1], &channels) || !integer(a[2], &k_pad) || !integer(a[3], &timestep) ||
      !integer(a[4], &layout) || !norm_args(a + 5, &x) || !tensor(a[12], &xq))
    return nullptr;
  if (x.C != channels && !fail("X has the grouping's channels")) return nullptr;
  const c10::cuda::CUDAGuard on(x.x.device());
  if (!stream_on(a[14], x.x, &st)) return nullptr;
  const int64_t rows = static_cast<int64_t>(x.B) * x.P;
  if (!xq.defined()) {
    xq = empty({rows, k_pad}, at::kByte, x.x);
    on_stream(xq, a[14], st);
  }
  if ((!xq.is_cuda() || xq.device() != x.x.device() || xq.scalar_type() != at::kByte || xq.dim() != 2 || xq.size(0) != rows ||
       xq.size(1) != k_pad || !xq.is_contiguous()) &&
      !fail("out is a contiguous uint8 tensor [B * P, K_pad] on X's device"))
    return nullptr;
  if (rows == 0) return output(a[12], xq);
  dgq_status rc;
  if (!norm_workspace(a[13], x, 1, a[14], st, &ws, &rc)) return nullptr;
  if (rc != DGQ_OK) return status(rc);
  const int type = dtype_of(x.x);
  void *p_add = ptr(x.add), *p_ws = ptr(ws), *p_xq = ptr(xq);
  const float *p_gamma = ptr<float>(x.gamma), *p_beta = ptr<float>(x.beta);
  const size_t bytes = ws.defined() ? ws.nbytes() : 0;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_group_norm_quantize(static_cast<const dgq_groups*>(g), timestep, layout, &x.rx, p_add, x.ld_add, p_gamma, p_beta, type, x.B, x.P,
                               x.n_groups, x.eps, x.act, p_xq, p_ws, bytes, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return output(a[12], xq);
}

// (weight, N, K, X, act, bias | None, out | None, stream) -> Y
PyObject* linear_few(PyObject* const* a, Py_ssize_t n) {
  void *st, *w;
  int n_out, k, act, m;
  at::Tensor x, bias, y;
  if (!arity(n, 8) || !handle(a[0], &w) || !integer(a[1], &n_out) || !integer(a[2], &k) || !tensor(a[3], &x) || !integer(a[4], &act) ||
      !tensor(a[5], &bias) || !tensor(a[6], &y))
    return nullptr;
  if ((!x.defined() || !x.is_cuda() || x.dim() != 2 || (x.scalar_type() != at::kHalf && x.scalar_type() != at::kBFloat16) || x.size(1) != k ||
       (k > 1 && x.stride(1) != 1)) &&
      !fail("X is a CUDA fp16 or bf16 matrix [M, K] with contiguous rows and the weight's K"))
    return nullptr;
  if (bias.defined() && (!bias.is_cuda() || bias.device() != x.device() || bias.scalar_type() != x.scalar_type() || !bias.is_contiguous() ||
                         bias.numel() != n_out) &&
      !fail("bias is a contiguous tensor [N] of X's type and device"))
    return nullptr;
  if (!fits(x.size(0), &m)) return nullptr;
  const c10::cuda::CUDAGuard on(x.device());
  if (!stream_on(a[7], x, &st)) return nullptr;
  if (!y.defined()) {
    y = empty({m, n_out}, x.scalar_type(), x);
    on_stream(y, a[7], st);
  }
  if ((!y.is_cuda() || y.device() != x.device() || y.scalar_type() != x.scalar_type() || y.dim() != 2 || y.size(0) != m || y.size(1) != n_out ||
       (n_out > 1 && y.stride(1) != 1)) &&
      !fail("out is a matrix [M, N] of X's type and device with contiguous rows"))
    return nullptr;
  if (m == 0) return output(a[6], y);
  const int type = dtype_of(x);
  const int64_t ldx = x.stride(0), ldy = y.stride(0);
  void *p_x = ptr(x), *p_bias = ptr(bias), *p_y = ptr(y);
  dgq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dgq_linear_few(static_cast<const dgq_few_weight*>(w), p_x, ldx, type, m, act, p_bias, p_y, ldy, st);
  Py_END_ALLOW_THREADS
  if (rc != DGQ_OK) return status(rc);
  return output(a[6], y);
}

template <PyObject* (*BODY)(PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(entry<BODY>)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<quantize_act>("quantize_act"), method<linear>("linear"),
                         method<cross_attn_logq>("cross_attn_logq"), method<self_attn_logq>("self_attn_logq"),
                         method<encoder_attn>("encoder_attn"), method<cached_attn>("cached_attn"), method<kv_plan>("kv_plan"),
                         method<kv_write>("kv_write"), method<kv_read>("kv_read"), method<group_norm>("group_norm"),
                         method<group_norm_quantize>("group_norm_quantize"), method<linear_few>("linear_few"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
