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
// These two make the results that are None: a call through ctypes takes the host 12 us, and the GPU as little as 2.5.
// Operands that may be missing are None; stream is None (the current one) or a cudaStream_t as an integer.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

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

PyMethodDef methods[] = {
    {"set_entry", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(set_entry)), METH_FASTCALL, "address of a library entry point"},
    {"layer", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(layer)), METH_FASTCALL, "one whole-layer call"},
    {"set_operator", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(set_operator)), METH_FASTCALL, "address of an operator"},
    {"product", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(product)), METH_FASTCALL, "one product of the operators"},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm)), METH_FASTCALL, "one norm"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torq_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torq_binding() { return PyModule_Create(&module); }
