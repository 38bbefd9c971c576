// The marshalling of the layer calls and of the operators around the layer in native code (a CPython extension).  A layer of a few tokens takes the GPU
// 6 us, its two kernel launches take the host 4.2 (both measured); checking seven tensors, reading their addresses and
// converting fifteen arguments in Python took another 5.7.  Nothing is computed here, and nothing is kept between calls
// but the addresses of the library's entry points.
//
//   set_entry(kind, address)   kind 0..3: torq_rotated_linear, _mxint4, _structured, _nvfp4
//   layer(kind, X, R, R_intra, Wq, Ws, Y, workspace, dbg_codes, dbg_scales, stream[, x_scale, w_scale])
//     -> the library's status, or -1 when an operand is not what the call takes (the caller then finds out which).
//   set_operator(kind, address)   kind 0..2: torq_{mxfp4,nvfp4,mxint4}_matvec, 3..5: _gated_matvec, 6..8: _gated_gemm, 9, 10:
//                                 torq_add_rmsnorm, _mxfp8, 11: torq_matvec_workspace_bytes
//   product(kind, A, As, W, Ws, Y, float32 out, stream, a_scale, w_scale, workspace) -> Y, or a status or -1 as above
//   norm(mxfp8, X, weight, residual, eps, out, out_scales, residual_out, stream) -> the tuple of results, or a status or -1
//   set_kv(op, fmt, address)   op 0..4: torq_{mxfp4,nvfp4,mxint4}_kv_append, _read, _attention, _weights, _evict; 5: torq_kv_attention_workspace_bytes
//   kv_append(fmt, pages, table, lengths, K, V, starts, k_scale, v_scale, stream) -> a status or -1
//   kv_read(fmt, pages, table, lengths, head_dim, tokens, starts, k_scale, v_scale, float32 out, stream) -> (K, V)
//   kv_attention(fmt, pages, table, lengths, Q, starts, k_scale, v_scale, scale, softcap, slopes, window, prefix, first, out, lse wanted, workspace,
//                stream) -> out or (out, lse)
//   kv_weights(fmt, pages, table, lengths, Q, lse, weights, starts, k_scale, scale, softcap, slopes, window, prefix, first, weights_out, stream)
//     -> a status or -1
//   kv_evict(fmt, pages, table, lengths, head_dim, weights, new_table, keep, recent, stream) -> (lengths, kept)
// Those with results make the ones that are None: a call through ctypes takes the host 12 us, and the GPU as little as 2.5.
// Operands that may be missing are None; stream is None (the current one) or a cudaStream_t as an integer.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <cmath>

#include "../../include/torq.h"

namespace {

using LayerFn = decltype(&torq_rotated_linear);
using LayerNvFn = decltype(&torq_rotated_linear_nvfp4);
constexpr int kNv = 3, kKinds = 4;
void* g_entry[kKinds] = {};

// Address of a contiguous CUDA tensor of `dtype`; None gives NULL where that is allowed.
bool operand(PyObject* o, at::ScalarType dtype, bool optional, void** out) {
  *out = nullptr;
  if (o == Py_None) return optional;
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != dtype || !t.is_cuda() || !t.is_contiguous()) return false;
  *out = t.data_ptr();
  return true;
}

// Scratch: any dtype; the caller counts a byte for each element.
bool scratch(PyObject* o, void** out, size_t* bytes) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || !t.is_contiguous()) return false;
  *out = t.data_ptr();
  *bytes = (size_t)t.numel();
  return true;
}

PyObject* set_entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const long kind = n == 2 ? PyLong_AsLong(a[0]) : -1;
  if (kind < 0 || kind >= kKinds) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "set_entry(kind, address)");
    return nullptr;
  }
  void* p = PyLong_AsVoidPtr(a[1]);
  if (PyErr_Occurred()) return nullptr;
  g_entry[kind] = p;
  Py_RETURN_NONE;
}

PyObject* layer(PyObject*, PyObject* const* a, Py_ssize_t n) try {
  const long kind = n >= 11 ? PyLong_AsLong(a[0]) : -1;
  if (kind < 0 || kind >= kKinds || n != (kind == kNv ? 13 : 11) || !g_entry[kind]) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "layer(): wrong arguments");
    return nullptr;
  }
  void *X, *R, *Ri, *Wq, *Ws, *ws, *dc, *ds;
  size_t ws_bytes;
  if (!operand(a[1], at::kBFloat16, false, &X) || !operand(a[2], at::kBFloat16, true, &R) ||
      !operand(a[3], at::kBFloat16, true, &Ri) || !operand(a[4], at::kByte, false, &Wq) || !operand(a[5], at::kByte, false, &Ws) ||
      !scratch(a[7], &ws, &ws_bytes) || !operand(a[8], at::kByte, true, &dc) || !operand(a[9], at::kByte, true, &ds) ||
      !THPVariable_Check(a[6]))
    return PyLong_FromLong(-1);
  const at::Tensor &x = THPVariable_Unpack(a[1]), &w = THPVariable_Unpack(a[4]), &y = THPVariable_Unpack(a[6]);
  const bool f32 = y.scalar_type() == at::kFloat;
  if (x.dim() != 2 || w.dim() < 1 || !y.is_cuda() || !y.is_contiguous() || (!f32 && y.scalar_type() != at::kBFloat16) ||
      y.numel() < x.size(0) * w.size(0))
    return PyLong_FromLong(-1);
  void* stream = a[10] == Py_None ? (void*)c10::cuda::getCurrentCUDAStream().stream() : PyLong_AsVoidPtr(a[10]);
  if (PyErr_Occurred()) return nullptr;
  const int64_t M = x.size(0), d = x.size(1), N = w.size(0);
  const torq_dtype dt = f32 ? TORQ_F32 : TORQ_BF16;
  void* yp = y.data_ptr();
  torq_status rc;
  if (kind == kNv) {
    const double xs = PyFloat_AsDouble(a[11]), wsc = PyFloat_AsDouble(a[12]);
    if (PyErr_Occurred()) return nullptr;
    Py_BEGIN_ALLOW_THREADS;                              // a launch may wait for room in the stream's queue
    rc = reinterpret_cast<LayerNvFn>(g_entry[kind])(X, R, Ri, (float)xs, Wq, Ws, (float)wsc, M, d, N, yp, dt, ws, ws_bytes, dc, ds, stream);
    Py_END_ALLOW_THREADS;
  } else {
    Py_BEGIN_ALLOW_THREADS;
    rc = reinterpret_cast<LayerFn>(g_entry[kind])(X, R, Ri, Wq, Ws, M, d, N, yp, dt, ws, ws_bytes, dc, ds, stream);
    Py_END_ALLOW_THREADS;
  }
  return PyLong_FromLong((long)rc);
} catch (const std::exception&) {                        // a tensor without storage, for instance
  return PyLong_FromLong(-1);
}

// ---- the operators around the layer ----------------------------------------------------------------------------------
enum { kNorm = 9, kNormMx = 10, kMatvecWorkspace = 11, kOperators = 12 };
void* g_operator[kOperators] = {};

PyObject* set_operator(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const long kind = n == 2 ? PyLong_AsLong(a[0]) : -1;
  if (kind < 0 || kind >= kOperators) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "set_operator(kind, address)");
    return nullptr;
  }
  void* p = PyLong_AsVoidPtr(a[1]);
  if (PyErr_Occurred()) return nullptr;
  g_operator[kind] = p;
  Py_RETURN_NONE;
}

bool is_cuda(PyObject* o) { return THPVariable_Check(o) && THPVariable_Unpack(o).is_cuda(); }
// A contiguous tensor of the current device; null where it is none.
const at::Tensor* plain(PyObject* o, c10::DeviceIndex device) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.device().index() == device && t.is_contiguous() ? &t : nullptr;
}
bool is_float(const at::Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
torq_dtype dtype_of(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? TORQ_F32 : TORQ_BF16; }
bool is_matrix(const at::Tensor& t, int64_t rows, int64_t cols) { return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols; }
// Scale bytes of [rows, k] with `block` elements to a scale, in whole tiles.
int64_t scale_bytes(int64_t rows, int64_t k, int64_t block) { return (rows + 127) / 128 * ((k / block + 3) / 4) * 512; }
// What a call makes belongs to the current stream's pool; where another stream is given, the allocator has to know that it uses it.
void used_by(const at::Tensor& t, PyObject* stream, void* handle) {
  if (stream != Py_None && t.defined()) t.record_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(handle), t.device().index()));
}
void* stream_of(PyObject* o) { return o == Py_None ? (void*)c10::cuda::getCurrentCUDAStream().stream() : PyLong_AsVoidPtr(o); }

PyObject* product(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const long kind = n == 11 ? PyLong_AsLong(a[0]) : -1;
  if (kind < 0 || kind >= kNorm || !g_operator[kind] || !g_operator[kMatvecWorkspace]) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "product(): wrong arguments");
    return nullptr;
  }
  const bool gemm = kind >= 6, gated = kind >= 3, nv = kind % 3 == 1;
  const int64_t per_byte = kind == 8 ? 1 : 2, block = nv ? 16 : 32;
  if (!is_cuda(a[1])) return PyLong_FromLong(-1);        // there may be no device to ask for
  const c10::DeviceIndex device = c10::cuda::current_device();
  const at::Tensor *A = plain(a[1], device), *As = gemm ? plain(a[2], device) : nullptr, *W = plain(a[3], device), *Ws = plain(a[4], device);
  if (!A || (gemm && !As) || !W || !Ws || A->scalar_type() != (gemm ? at::kByte : at::kBFloat16) || W->scalar_type() != at::kByte ||
      Ws->scalar_type() != at::kByte || A->dim() != 2 || W->dim() != 2)
    return PyLong_FromLong(-1);
  const int64_t M = A->size(0), rows = W->size(0), K = W->size(1) * per_byte, N = gated ? rows / 2 : rows;
  if (A->size(1) * (gemm ? per_byte : 1) != K || (gated && rows % 2) || Ws->numel() < scale_bytes(rows, K, block) ||
      (gemm && (As->scalar_type() != at::kByte || As->numel() < scale_bytes(M, K, block))))
    return PyLong_FromLong(-1);
  at::Tensor Y;
  if (a[5] == Py_None) {
    Y = at::empty({M, N}, A->options().dtype(PyObject_IsTrue(a[6]) ? at::kFloat : at::kBFloat16));
  } else {
    const at::Tensor* y = plain(a[5], device);
    if (!y || !is_float(*y) || !is_matrix(*y, M, N)) return PyLong_FromLong(-1);
    Y = *y;
  }
  at::Tensor scratch;
  size_t scratch_bytes = 0;
  if (!gemm && a[10] != Py_None) {
    const at::Tensor* t = plain(a[10], device);
    if (!t) return PyLong_FromLong(-1);
    scratch = *t;
    scratch_bytes = (size_t)t->nbytes();
  } else if (!gemm) {
    scratch_bytes = reinterpret_cast<decltype(&torq_matvec_workspace_bytes)>(g_operator[kMatvecWorkspace])(M, N, K);
    if (scratch_bytes) scratch = at::empty({(int64_t)scratch_bytes}, W->options());
  }
  void* stream = stream_of(a[7]);
  if (PyErr_Occurred()) return nullptr;
  used_by(scratch, a[7], stream);
  if (a[5] == Py_None) used_by(Y, a[7], stream);
  const float a_scale = nv ? (float)PyFloat_AsDouble(a[8]) : 0.f, w_scale = nv ? (float)PyFloat_AsDouble(a[9]) : 0.f;
  if (PyErr_Occurred()) return nullptr;
  const void *ap = A->data_ptr(), *asp = gemm ? As->data_ptr() : nullptr, *wp = W->data_ptr(), *wsp = Ws->data_ptr();
  void *yp = Y.data_ptr(), *f = g_operator[kind], *sp = scratch.defined() ? scratch.data_ptr() : nullptr;
  const torq_dtype dt = dtype_of(Y);
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;                                // a launch may wait for room in the stream's queue
  if (gemm && nv) rc = reinterpret_cast<decltype(&torq_nvfp4_gated_gemm)>(f)(ap, asp, a_scale, wp, wsp, w_scale, M, N, K, yp, dt, stream);
  else if (gemm) rc = reinterpret_cast<decltype(&torq_mxfp4_gated_gemm)>(f)(ap, asp, wp, wsp, M, N, K, yp, dt, stream);
  else if (nv) rc = reinterpret_cast<decltype(&torq_nvfp4_matvec)>(f)(ap, wp, wsp, w_scale, M, N, K, yp, dt, sp, scratch_bytes, stream);
  else rc = reinterpret_cast<decltype(&torq_mxfp4_matvec)>(f)(ap, wp, wsp, M, N, K, yp, dt, sp, scratch_bytes, stream);
  Py_END_ALLOW_THREADS;
  if (rc != TORQ_OK) return PyLong_FromLong((long)rc);
  if (a[5] == Py_None) return THPVariable_Wrap(std::move(Y));
  Py_INCREF(a[5]);
  return a[5];
  END_HANDLE_TH_ERRORS
}

PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const int mx = n == 9 ? PyObject_IsTrue(a[0]) : -1;
  if (mx < 0 || !g_operator[kNorm] || !g_operator[kNormMx]) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "norm(): wrong arguments");
    return nullptr;
  }
  if (!is_cuda(a[1])) return PyLong_FromLong(-1);        // there may be no device to ask for
  const c10::DeviceIndex device = c10::cuda::current_device();
  const at::Tensor *X = plain(a[1], device), *w = plain(a[2], device), *R = a[3] == Py_None ? nullptr : plain(a[3], device);
  if (!X || !w || !is_float(*X) || X->dim() != 2 || w->scalar_type() != at::kBFloat16 || w->dim() != 1 || w->size(0) != X->size(1) ||
      (a[3] != Py_None && (!R || !is_float(*R) || !is_matrix(*R, X->size(0), X->size(1)))) || (a[3] == Py_None && a[7] != Py_None))
    return PyLong_FromLong(-1);
  const int64_t M = X->size(0), d = X->size(1), scales = scale_bytes(M, d, 32);
  at::Tensor out, sf, h;
  const at::ScalarType type = mx ? at::kByte : at::kBFloat16;
  if (a[5] == Py_None) {
    out = at::empty({M, d}, X->options().dtype(type));
  } else {
    const at::Tensor* t = plain(a[5], device);
    if (!t || t->scalar_type() != type || !is_matrix(*t, M, d)) return PyLong_FromLong(-1);
    out = *t;
  }
  if (mx && a[6] == Py_None) {
    sf = at::empty({scales}, X->options().dtype(at::kByte));
  } else if (mx) {
    const at::Tensor* t = plain(a[6], device);
    if (!t || t->scalar_type() != at::kByte || t->numel() < scales) return PyLong_FromLong(-1);
    sf = *t;
  }
  if (R && a[7] == Py_None) {
    h = at::empty_like(*R);
  } else if (R) {
    const at::Tensor* t = plain(a[7], device);
    if (!t || t->scalar_type() != R->scalar_type() || !is_matrix(*t, M, d)) return PyLong_FromLong(-1);
    h = *t;
  }
  const float eps = (float)PyFloat_AsDouble(a[4]);
  void* stream = stream_of(a[8]);
  if (PyErr_Occurred()) return nullptr;
  if (a[5] == Py_None) used_by(out, a[8], stream);
  if (mx && a[6] == Py_None) used_by(sf, a[8], stream);
  if (R && a[7] == Py_None) used_by(h, a[8], stream);
  const void *xp = X->data_ptr(), *wp = w->data_ptr(), *rp = R ? R->data_ptr() : nullptr;
  void *op = out.data_ptr(), *sp = mx ? sf.data_ptr() : nullptr, *hp = R ? h.data_ptr() : nullptr;
  const torq_dtype xt = dtype_of(*X), rt = R ? dtype_of(*R) : TORQ_BF16;
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;
  if (mx) rc = reinterpret_cast<decltype(&torq_add_rmsnorm_mxfp8)>(g_operator[kNormMx])(xp, xt, rp, hp, rt, wp, eps, M, d, op, sp, stream);
  else rc = reinterpret_cast<decltype(&torq_add_rmsnorm)>(g_operator[kNorm])(xp, xt, rp, hp, rt, wp, eps, M, d, op, stream);
  Py_END_ALLOW_THREADS;
  if (rc != TORQ_OK) return PyLong_FromLong((long)rc);
  auto give = [](PyObject* o, at::Tensor& t) {
    if (o == Py_None) return THPVariable_Wrap(std::move(t));
    Py_INCREF(o);
    return o;
  };
  PyObject* r = PyTuple_New(1 + (mx ? 1 : 0) + (R ? 1 : 0));
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, give(a[5], out));
  if (mx) PyTuple_SET_ITEM(r, 1, give(a[6], sf));
  if (R) PyTuple_SET_ITEM(r, 1 + (mx ? 1 : 0), give(a[7], h));
  return r;
  END_HANDLE_TH_ERRORS
}

// ---- the 4-bit key/value cache -----------------------------------------------------------------------------------------
enum { kKvAppend, kKvRead, kKvAttention, kKvWeights, kKvEvict, kKvWorkspace, kKvOps };
void* g_kv[kKvOps][3] = {};

PyObject* set_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const long op = n == 3 ? PyLong_AsLong(a[0]) : -1, fmt = n == 3 ? PyLong_AsLong(a[1]) : -1;
  if (op < 0 || op >= kKvOps || fmt < 0 || fmt > 2) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "set_kv(op, fmt, address)");
    return nullptr;
  }
  void* p = PyLong_AsVoidPtr(a[2]);
  if (PyErr_Occurred()) return nullptr;
  g_kv[op][fmt] = p;
  Py_RETURN_NONE;
}

// The format of a call with `count` arguments of which `n` came; -1 with an exception.
long kv_format(PyObject* const* a, Py_ssize_t n, Py_ssize_t count, int op, const char* name) {
  const long fmt = n == count ? PyLong_AsLong(a[0]) : -1;
  if (fmt < 0 || fmt > 2 || !g_kv[op][fmt] || !g_kv[kKvWorkspace][0]) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s(): wrong arguments", name);
    return -1;
  }
  return fmt;
}
// A contiguous tensor of the current device and of that type; where it may be missing, None gives null.
bool typed(PyObject* o, c10::DeviceIndex device, at::ScalarType type, bool optional, const at::Tensor** t) {
  *t = nullptr;
  if (o == Py_None) return optional;
  *t = plain(o, device);
  return *t && (*t)->scalar_type() == type;
}
// [tokens, heads, dim] whose rows may lie apart, and their distance.
bool kv_rows(PyObject* o, c10::DeviceIndex device, const at::Tensor** t, int64_t* stride) {
  if (!THPVariable_Check(o)) return false;
  *t = &THPVariable_Unpack(o);
  const at::Tensor& x = **t;
  if (!x.is_cuda() || x.device().index() != device || x.dim() != 3) return false;
  const int64_t tokens = x.size(0), heads = x.size(1), dim = x.size(2);
  if ((x.stride(2) != 1 && dim > 1) || (x.stride(1) != dim && heads > 1) || (x.stride(0) < heads * dim && tokens > 1)) return false;
  *stride = tokens > 1 ? x.stride(0) : heads * dim;
  return true;
}
// What the cache of a call is made of; a[0..2] are pages, table, lengths.
bool kv_cache(PyObject* const* a, PyObject* starts, c10::DeviceIndex device, long fmt, int64_t dim, int64_t tokens, double k_scale, double v_scale,
              torq_kv_cache* c, const int32_t** starts_p) {
  const at::Tensor *pages, *table, *lengths, *st;
  if (!typed(a[0], device, at::kByte, false, &pages) || !typed(a[1], device, at::kInt, false, &table) ||
      !typed(a[2], device, at::kInt, false, &lengths) || !typed(starts, device, at::kInt, true, &st) || pages->dim() != 3 || table->dim() != 2 ||
      (dim != 64 && dim != 128 && dim != 256))
    return false;
  const int64_t batch = table->size(0), one = 2 * (dim / 2 + dim / (fmt == 1 ? 16 : 32));
  if (lengths->dim() != 1 || lengths->size(0) != batch || (st ? st->dim() != 1 || st->size(0) != batch + 1 : tokens != batch) ||
      pages->size(2) % one)
    return false;
  *c = {pages->data_ptr(), static_cast<const int32_t*>(table->data_ptr()), static_cast<const int32_t*>(lengths->data_ptr()), pages->size(0),
        pages->size(2) / one, pages->size(1), dim, batch, table->size(1), (float)k_scale, (float)v_scale};
  *starts_p = st ? static_cast<const int32_t*>(st->data_ptr()) : nullptr;
  return true;
}
// scale, softcap, slopes, window, prefix, first
bool kv_scoring(PyObject* const* a, c10::DeviceIndex device, int64_t dim, int64_t heads, int64_t batch, int64_t tokens, torq_kv_scoring* s) {
  const at::Tensor *slopes, *prefix, *first;
  if (!typed(a[2], device, at::kFloat, true, &slopes) || !typed(a[4], device, at::kInt, true, &prefix) || !typed(a[5], device, at::kInt, true, &first))
    return false;
  if ((slopes && (slopes->dim() != 1 || slopes->size(0) != heads)) || (prefix && (prefix->dim() != 1 || prefix->size(0) != batch)) ||
      (first && (first->dim() != 1 || first->size(0) != tokens)))
    return false;
  s->scale = a[0] == Py_None ? (float)(1.0 / std::sqrt((double)dim)) : (float)PyFloat_AsDouble(a[0]);
  s->softcap = (float)PyFloat_AsDouble(a[1]);
  s->slopes = slopes ? static_cast<const float*>(slopes->data_ptr()) : nullptr;
  s->window = PyLong_AsLongLong(a[3]);
  s->prefix = prefix ? static_cast<const int32_t*>(prefix->data_ptr()) : nullptr;
  s->first = first ? static_cast<const int32_t*>(first->data_ptr()) : nullptr;
  return true;
}

PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const long fmt = kv_format(a, n, 10, kKvAppend, "kv_append");
  if (fmt < 0) return nullptr;
  if (!is_cuda(a[1])) return PyLong_FromLong(-1);        // there may be no device to ask for
  const c10::DeviceIndex device = c10::cuda::current_device();
  const at::Tensor *K, *V;
  int64_t ks, vs;
  torq_kv_cache c;
  const int32_t* starts;
  const double k_scale = PyFloat_AsDouble(a[7]), v_scale = PyFloat_AsDouble(a[8]);
  if (PyErr_Occurred()) return nullptr;
  if (!kv_rows(a[4], device, &K, &ks) || !kv_rows(a[5], device, &V, &vs) || !is_float(*K) || V->scalar_type() != K->scalar_type() ||
      V->sizes() != K->sizes() || !kv_cache(a + 1, a[6], device, fmt, K->size(2), K->size(0), k_scale, v_scale, &c, &starts) ||
      K->size(1) != c.kv_heads)
    return PyLong_FromLong(-1);
  void* stream = stream_of(a[9]);
  if (PyErr_Occurred()) return nullptr;
  const void *k = K->data_ptr(), *v = V->data_ptr();
  const torq_dtype dt = dtype_of(*K);
  const int64_t tokens = K->size(0);
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = reinterpret_cast<decltype(&torq_mxfp4_kv_append)>(g_kv[kKvAppend][fmt])(&c, k, v, dt, ks, vs, starts, tokens, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong((long)rc);
  END_HANDLE_TH_ERRORS
}

PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const long fmt = kv_format(a, n, 11, kKvRead, "kv_read");
  if (fmt < 0) return nullptr;
  if (!is_cuda(a[1])) return PyLong_FromLong(-1);
  const c10::DeviceIndex device = c10::cuda::current_device();
  const int64_t dim = PyLong_AsLongLong(a[4]), tokens = PyLong_AsLongLong(a[5]);
  const double k_scale = PyFloat_AsDouble(a[7]), v_scale = PyFloat_AsDouble(a[8]);
  const int f32 = PyObject_IsTrue(a[9]);
  if (PyErr_Occurred()) return nullptr;
  torq_kv_cache c;
  const int32_t* starts;
  if (tokens < 1 || !kv_cache(a + 1, a[6], device, fmt, dim, tokens, k_scale, v_scale, &c, &starts)) return PyLong_FromLong(-1);
  const auto options = THPVariable_Unpack(a[1]).options().dtype(f32 ? at::kFloat : at::kBFloat16);
  at::Tensor K = at::empty({tokens, c.kv_heads, dim}, options), V = at::empty({tokens, c.kv_heads, dim}, options);
  void* stream = stream_of(a[10]);
  if (PyErr_Occurred()) return nullptr;
  used_by(K, a[10], stream);
  used_by(V, a[10], stream);
  void *k = K.data_ptr(), *v = V.data_ptr();
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = reinterpret_cast<decltype(&torq_mxfp4_kv_read)>(g_kv[kKvRead][fmt])(&c, starts, tokens, k, v, f32 ? TORQ_F32 : TORQ_BF16, stream);
  Py_END_ALLOW_THREADS;
  if (rc != TORQ_OK) return PyLong_FromLong((long)rc);
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(std::move(K)));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(std::move(V)));
  return r;
  END_HANDLE_TH_ERRORS
}

PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const long fmt = kv_format(a, n, 18, kKvAttention, "kv_attention");
  if (fmt < 0) return nullptr;
  if (!is_cuda(a[1])) return PyLong_FromLong(-1);
  const c10::DeviceIndex device = c10::cuda::current_device();
  const at::Tensor* Q;
  int64_t stride;
  torq_kv_cache c;
  torq_kv_scoring s;
  const int32_t* starts;
  const double k_scale = PyFloat_AsDouble(a[6]), v_scale = PyFloat_AsDouble(a[7]);
  if (PyErr_Occurred()) return nullptr;
  if (!kv_rows(a[4], device, &Q, &stride) || Q->scalar_type() != at::kBFloat16) return PyLong_FromLong(-1);
  const int64_t tokens = Q->size(0), heads = Q->size(1), dim = Q->size(2);
  if (!kv_cache(a + 1, a[5], device, fmt, dim, tokens, k_scale, v_scale, &c, &starts) || c.kv_heads < 1 || heads % c.kv_heads ||
      !kv_scoring(a + 8, device, dim, heads, c.batch, tokens, &s))
    return PyErr_Occurred() ? nullptr : PyLong_FromLong(-1);
  at::Tensor out, lse, scratch;
  if (a[14] == Py_None) {
    out = at::empty({tokens, heads, dim}, Q->options());
  } else {
    const at::Tensor* t = plain(a[14], device);
    if (!t || t->scalar_type() != at::kBFloat16 || t->sizes() != Q->sizes()) return PyLong_FromLong(-1);
    out = *t;
  }
  const int want = PyObject_IsTrue(a[15]);
  if (want) lse = at::empty({tokens, heads}, Q->options().dtype(at::kFloat));
  size_t bytes;
  if (a[16] == Py_None) {
    bytes = reinterpret_cast<decltype(&torq_kv_attention_workspace_bytes)>(g_kv[kKvWorkspace][0])(tokens, c.batch, heads, c.kv_heads, dim);
    if (bytes) scratch = at::empty({(int64_t)bytes}, Q->options().dtype(at::kByte));
  } else {
    const at::Tensor* t = plain(a[16], device);
    if (!t) return PyLong_FromLong(-1);
    scratch = *t;
    bytes = (size_t)t->nbytes();
  }
  void* stream = stream_of(a[17]);
  if (PyErr_Occurred()) return nullptr;
  if (a[14] == Py_None) used_by(out, a[17], stream);
  used_by(lse, a[17], stream);
  used_by(scratch, a[17], stream);
  const void* q = Q->data_ptr();
  void *o = out.data_ptr(), *w = scratch.defined() ? scratch.data_ptr() : nullptr;
  float* y = want ? static_cast<float*>(lse.data_ptr()) : nullptr;
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = reinterpret_cast<decltype(&torq_mxfp4_kv_attention)>(g_kv[kKvAttention][fmt])(&c, &s, q, stride, heads, starts, tokens, o, y, w, bytes, stream);
  Py_END_ALLOW_THREADS;
  if (rc != TORQ_OK) return PyLong_FromLong((long)rc);
  PyObject* first = a[14];
  if (first == Py_None) first = THPVariable_Wrap(std::move(out));
  else Py_INCREF(first);
  if (!want) return first;
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, first);
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(std::move(lse)));
  return r;
  END_HANDLE_TH_ERRORS
}

PyObject* kv_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const long fmt = kv_format(a, n, 17, kKvWeights, "kv_weights");
  if (fmt < 0) return nullptr;
  if (!is_cuda(a[1])) return PyLong_FromLong(-1);
  const c10::DeviceIndex device = c10::cuda::current_device();
  const at::Tensor *Q, *lse, *w, *o;
  int64_t stride;
  torq_kv_cache c;
  torq_kv_scoring s;
  const int32_t* starts;
  const double k_scale = PyFloat_AsDouble(a[8]);
  if (PyErr_Occurred()) return nullptr;
  if (!kv_rows(a[4], device, &Q, &stride) || Q->scalar_type() != at::kBFloat16) return PyLong_FromLong(-1);
  const int64_t tokens = Q->size(0), heads = Q->size(1), dim = Q->size(2);
  if (!kv_cache(a + 1, a[7], device, fmt, dim, tokens, k_scale, 1.0, &c, &starts) || c.kv_heads < 1 || heads % c.kv_heads ||
      !typed(a[5], device, at::kFloat, false, &lse) || !typed(a[6], device, at::kFloat, false, &w) || !typed(a[15], device, at::kFloat, true, &o) ||
      !is_matrix(*lse, tokens, heads) || !kv_scoring(a + 9, device, dim, heads, c.batch, tokens, &s))
    return PyErr_Occurred() ? nullptr : PyLong_FromLong(-1);
  if (!o) o = w;
  for (const at::Tensor* t : {w, o})
    if (t->dim() != 3 || t->size(0) != c.num_pages || t->size(1) != c.kv_heads || t->size(2) != c.page_tokens) return PyLong_FromLong(-1);
  void* stream = stream_of(a[16]);
  if (PyErr_Occurred()) return nullptr;
  const void* q = Q->data_ptr();
  const float *y = static_cast<const float*>(lse->data_ptr()), *from = static_cast<const float*>(w->data_ptr());
  float* to = static_cast<float*>(o->data_ptr());
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = reinterpret_cast<decltype(&torq_mxfp4_kv_weights)>(g_kv[kKvWeights][fmt])(&c, &s, q, stride, heads, starts, tokens, y, from, to, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong((long)rc);
  END_HANDLE_TH_ERRORS
}

PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const long fmt = kv_format(a, n, 10, kKvEvict, "kv_evict");
  if (fmt < 0) return nullptr;
  if (!is_cuda(a[1]) || !THPVariable_Check(a[2]) || THPVariable_Unpack(a[2]).dim() != 2) return PyLong_FromLong(-1);
  const c10::DeviceIndex device = c10::cuda::current_device();
  const int64_t dim = PyLong_AsLongLong(a[4]), keep = PyLong_AsLongLong(a[7]), recent = PyLong_AsLongLong(a[8]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *w, *to;
  torq_kv_cache c;
  const int32_t* starts;
  if (!kv_cache(a + 1, Py_None, device, fmt, dim, THPVariable_Unpack(a[2]).size(0), 1.0, 1.0, &c, &starts) || !typed(a[5], device, at::kFloat, false, &w) ||
      !typed(a[6], device, at::kInt, false, &to) || to->dim() != 2 || to->size(0) != c.batch || w->dim() != 3 || w->size(0) != c.num_pages ||
      w->size(1) != c.kv_heads || w->size(2) != c.page_tokens || keep < 1)
    return PyLong_FromLong(-1);
  at::Tensor lengths = at::empty({c.batch}, to->options()), kept = at::empty({c.batch, c.kv_heads, keep}, to->options());
  void* stream = stream_of(a[9]);
  if (PyErr_Occurred()) return nullptr;
  used_by(lengths, a[9], stream);
  used_by(kept, a[9], stream);
  float* wp = static_cast<float*>(w->data_ptr());
  const int32_t* tp = static_cast<const int32_t*>(to->data_ptr());
  int32_t *lp = static_cast<int32_t*>(lengths.data_ptr()), *kp = static_cast<int32_t*>(kept.data_ptr());
  const int64_t width = to->size(1);
  torq_status rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = reinterpret_cast<decltype(&torq_mxfp4_kv_evict)>(g_kv[kKvEvict][fmt])(&c, wp, tp, width, keep, recent, lp, kp, stream);
  Py_END_ALLOW_THREADS;
  if (rc != TORQ_OK) return PyLong_FromLong((long)rc);
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(std::move(lengths)));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(std::move(kept)));
  return r;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"set_entry", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(set_entry)), METH_FASTCALL, "address of a library entry point"},
    {"layer", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(layer)), METH_FASTCALL, "one whole-layer call"},
    {"set_operator", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(set_operator)), METH_FASTCALL, "address of an operator"},
    {"product", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(product)), METH_FASTCALL, "one product of the operators"},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm)), METH_FASTCALL, "one norm"},
    {"set_kv", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(set_kv)), METH_FASTCALL, "address of an entry point of the cache"},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_append)), METH_FASTCALL, "new tokens into the cache"},
    {"kv_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_read)), METH_FASTCALL, "tokens of the cache"},
    {"kv_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_attention)), METH_FASTCALL, "attention over the cache"},
    {"kv_weights", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_weights)), METH_FASTCALL, "account of attention weight"},
    {"kv_evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_evict)), METH_FASTCALL, "eviction by account"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torq_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torq_binding() { return PyModule_Create(&module); }
