"""Thin binding over the C-ABI library (include/torq.h): ctypes, and for the whole-layer calls a native extension.
Argument marshalling only: every step of the path runs in the CUDA kernels; PyTorch provides device memory and streams.
There is no fallback: a missing library or a non-zero status raises."""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings

import torch

from . import build as _build

TORQ_F32, TORQ_BF16 = 0, 1
_STATUS = {0: "TORQ_OK", 1: "TORQ_ERR_NULL", 2: "TORQ_ERR_SHAPE", 3: "TORQ_ERR_ALIGN", 4: "TORQ_ERR_ARCH",
           5: "TORQ_ERR_LAUNCH", 6: "TORQ_ERR_TIMEOUT", 7: "TORQ_ERR_WORKSPACE", 8: "TORQ_ERR_PAGE"}
_lib_handle = None


class _KvCache(ctypes.Structure):                # torq_kv_cache
    _fields_ = [("pages", ctypes.c_void_p), ("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                *((n, ctypes.c_int64) for n in ("num_pages", "page_tokens", "kv_heads", "head_dim", "batch", "table_width")),
                ("k_tensor_scale", ctypes.c_float), ("v_tensor_scale", ctypes.c_float)]


class _KvScoring(ctypes.Structure):              # torq_kv_scoring
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("window", ctypes.c_int64),
                ("prefix", ctypes.c_void_p), ("first", ctypes.c_void_p)]


class TorqError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_STATUS.get(code, code)}")


def lib() -> ctypes.CDLL:
    """Loads (building first if the binary is absent or stale and nvcc is available)."""
    global _lib_handle
    if _lib_handle is not None:
        return _lib_handle
    path = _build.LIB_PATH
    if _build.needs_build():
        _build.build_library()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing; run paper_2605_19561_b200/build.py")
    L = ctypes.CDLL(path)
    vp, i64, sz, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    L.torq_rotate_quantize.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp]
    L.torq_rotate_quantize.restype = ci
    L.torq_rotate_quantize_structured.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp]
    L.torq_rotate_quantize_structured.restype = ci
    L.torq_rotated_linear_structured.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, ci, vp, sz, vp, vp, vp]
    L.torq_rotated_linear_structured.restype = ci
    L.torq_mxfp4_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, ci, vp]
    L.torq_mxfp4_gemm.restype = ci
    L.torq_rotated_linear.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, ci, vp, sz, vp, vp, vp]
    L.torq_rotated_linear.restype = ci
    L.torq_rotated_linear_static.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, ci, vp]
    L.torq_rotated_linear_static.restype = ci
    L.torq_quantize_mxfp4.argtypes = [vp, ci, i64, i64, vp, vp, vp]
    L.torq_quantize_mxfp4.restype = ci
    L.torq_scales_bytes.argtypes = [i64, i64]
    L.torq_scales_bytes.restype = sz
    L.torq_scale_offset.argtypes = [i64, i64, i64]
    L.torq_scale_offset.restype = sz
    L.torq_workspace_bytes.argtypes = [i64, i64, i64]
    L.torq_workspace_bytes.restype = sz
    L.torq_swizzle_scales.argtypes = [vp, i64, i64, vp, vp]
    L.torq_swizzle_scales.restype = ci
    L.torq_merge_rotations.argtypes = [vp, vp, i64, vp, vp]
    L.torq_merge_rotations.restype = ci
    f32 = ctypes.c_float
    L.torq_merge_rotations_bf16.argtypes = [vp, vp, i64, vp, vp]
    L.torq_merge_rotations_bf16.restype = ci
    L.torq_prepare_weights_workspace_bytes.argtypes = [i64, i64]
    L.torq_prepare_weights_workspace_bytes.restype = sz
    L.torq_prepare_weights.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp, sz, vp]
    L.torq_prepare_weights.restype = ci
    L.torq_prepare_weights_nvfp4.argtypes = [vp, vp, vp, i64, i64, vp, vp, ctypes.POINTER(ctypes.c_float), vp, sz, vp]
    L.torq_prepare_weights_nvfp4.restype = ci
    L.torq_prepare_weights_mxint4.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp, vp, sz, vp]
    L.torq_prepare_weights_mxint4.restype = ci
    L.torq_nvfp4_scales_bytes.argtypes = [i64, i64]
    L.torq_nvfp4_scales_bytes.restype = sz
    L.torq_nvfp4_workspace_bytes.argtypes = [i64, i64, i64]
    L.torq_nvfp4_workspace_bytes.restype = sz
    L.torq_expand_intra16.argtypes = [vp, i64, vp, vp]
    L.torq_expand_intra16.restype = ci
    L.torq_quantize_nvfp4.argtypes = [vp, ci, i64, i64, f32, vp, vp, vp]
    L.torq_quantize_nvfp4.restype = ci
    L.torq_rotate_quantize_nvfp4.argtypes = [vp, vp, vp, i64, i64, f32, vp, vp, vp]
    L.torq_rotate_quantize_nvfp4.restype = ci
    L.torq_rotate_quantize_structured_nvfp4.argtypes = [vp, vp, vp, i64, i64, f32, vp, vp, vp]
    L.torq_rotate_quantize_structured_nvfp4.restype = ci
    L.torq_nvfp4_gemm.argtypes = [vp, vp, f32, vp, vp, f32, i64, i64, i64, vp, ci, vp]
    L.torq_nvfp4_gemm.restype = ci
    L.torq_rotated_linear_nvfp4.argtypes = [vp, vp, vp, f32, vp, vp, f32, i64, i64, i64, vp, ci, vp, sz, vp, vp, vp]
    L.torq_rotated_linear_nvfp4.restype = ci
    L.torq_mxint4_workspace_bytes.argtypes = [i64, i64, i64]
    L.torq_mxint4_workspace_bytes.restype = sz
    L.torq_quantize_mxint4.argtypes = [vp, ci, i64, i64, ci, vp, vp, vp]
    L.torq_quantize_mxint4.restype = ci
    L.torq_mxint4_expand.argtypes = [vp, i64, i64, vp, vp]
    L.torq_mxint4_expand.restype = ci
    L.torq_rotate_quantize_mxint4.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp]
    L.torq_rotate_quantize_mxint4.restype = ci
    L.torq_rotate_quantize_structured_mxint4.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp]
    L.torq_rotate_quantize_structured_mxint4.restype = ci
    L.torq_mxint4_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, ci, vp]
    L.torq_mxint4_gemm.restype = ci
    L.torq_rotated_linear_mxint4.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp, ci, vp, sz, vp, vp, vp]
    L.torq_rotated_linear_mxint4.restype = ci
    L.torq_add_rmsnorm.argtypes = [vp, ci, vp, vp, ci, vp, f32, i64, i64, vp, vp]
    L.torq_add_rmsnorm.restype = ci
    L.torq_add_rmsnorm_mxfp8.argtypes = [vp, ci, vp, vp, ci, vp, f32, i64, i64, vp, vp, vp]
    L.torq_add_rmsnorm_mxfp8.restype = ci
    for name in ("torq_mxfp4_matvec", "torq_mxint4_matvec", "torq_mxfp4_gated_matvec", "torq_mxint4_gated_matvec"):
        getattr(L, name).argtypes = [vp, vp, vp, i64, i64, i64, vp, ci, vp, sz, vp]
        getattr(L, name).restype = ci
    L.torq_matvec_workspace_bytes.argtypes = [i64, i64, i64]
    L.torq_matvec_workspace_bytes.restype = sz
    for name in ("torq_nvfp4_matvec", "torq_nvfp4_gated_matvec"):
        getattr(L, name).argtypes = [vp, vp, vp, f32, i64, i64, i64, vp, ci, vp, sz, vp]
        getattr(L, name).restype = ci
    for name in ("torq_mxfp4_gated_gemm", "torq_mxint4_gated_gemm"):
        getattr(L, name).argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, ci, vp]
        getattr(L, name).restype = ci
    L.torq_nvfp4_gated_gemm.argtypes = [vp, vp, f32, vp, vp, f32, i64, i64, i64, vp, ci, vp]
    L.torq_nvfp4_gated_gemm.restype = ci
    kc, ks = ctypes.POINTER(_KvCache), ctypes.POINTER(_KvScoring)
    for fmt in ("mxfp4", "nvfp4", "mxint4"):
        for name, args in (("append", [kc, vp, vp, ci, i64, i64, vp, i64, vp]), ("read", [kc, vp, i64, vp, vp, ci, vp]),
                           ("attention", [kc, ks, vp, i64, i64, vp, i64, vp, vp, vp, sz, vp]),
                           ("weights", [kc, ks, vp, i64, i64, vp, i64, vp, vp, vp, vp]), ("evict", [kc, vp, vp, i64, i64, i64, vp, vp, vp])):
            f = getattr(L, f"torq_{fmt}_kv_{name}")
            f.argtypes, f.restype = args, ci
    L.torq_kv_page_bytes.argtypes = [i64, i64, i64]
    L.torq_kv_page_bytes.restype = sz
    L.torq_kv_attention_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    L.torq_kv_attention_workspace_bytes.restype = sz
    L.torq_block_covariance.argtypes = [vp, i64, i64, vp, vp]
    L.torq_block_covariance.restype = ci
    L.torq_givens_equalize.argtypes = [vp, i64, ctypes.c_double, vp, vp, vp, vp]
    L.torq_givens_equalize.restype = ci
    L.torq_probe_fp4_peak.argtypes = [ci, ctypes.POINTER(ctypes.c_double), vp]
    L.torq_probe_fp4_peak.restype = ci
    L.torq_selftest_wait_timeout.argtypes = [ctypes.c_uint64, vp, vp]
    L.torq_selftest_wait_timeout.restype = ci
    L.torq_status_string.argtypes = [ci]
    L.torq_status_string.restype = ctypes.c_char_p
    L.torq_last_device_error.argtypes = [vp]
    L.torq_last_device_error.restype = ci
    L.torq_pair_tile_list.argtypes = [i64, i64, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), i64]
    L.torq_pair_tile_list.restype = i64
    L.torq_gemm_tile_list.argtypes = [i64, i64, i64, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), i64]
    L.torq_gemm_tile_list.restype = i64
    L.torq_launch_count.argtypes = []
    L.torq_launch_count.restype = i64
    _lib_handle = L
    return L


# The whole-layer calls go through the native binding (csrc/binding.cpp), which returns the library's status, or -1 for
# operands that it does not take: _refuse then says what is wrong with them.  It is built and loaded by the first such call;
# the library itself needs no compiler beside its own.  Where the binding cannot be had, the same call goes through ctypes.
_MXFP4, _MXINT4, _STRUCTURED, _NVFP4 = range(4)
_LAYER_ENTRIES = ("torq_rotated_linear", "torq_rotated_linear_mxint4", "torq_rotated_linear_structured",
                  "torq_rotated_linear_nvfp4")
_OPERATORS = (*(f"torq_{fmt}_{op}" for op in ("matvec", "gated_matvec", "gated_gemm") for fmt in ("mxfp4", "nvfp4", "mxint4")),
              "torq_add_rmsnorm", "torq_add_rmsnorm_mxfp8", "torq_matvec_workspace_bytes")


_KV_FORMATS = ("mxfp4", "nvfp4", "mxint4")


def _layer(*args):                               # until the first call has put the native function here
    global _layer
    _layer = _layer_native() or _layer_ctypes
    return _layer(*args)


def _layer_native():
    binding = _native_binding()
    return binding and binding.layer


_binding_module = None                           # None: not looked for yet; False: cannot be had


def _native_binding():
    global _binding_module
    if _binding_module is not None:
        return _binding_module or None
    L = lib()
    try:
        spec = importlib.util.spec_from_file_location(__package__ + "._torq_binding", _build.build_binding())
        binding = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(binding)
    except (ImportError, OSError, RuntimeError) as e:
        warnings.warn(f"the native binding of the layer calls is missing, they cost 5 us more on the host: {e}")
        _binding_module = False
        return None
    for set_address, names in ((binding.set_entry, _LAYER_ENTRIES), (binding.set_operator, _OPERATORS)):
        for kind, name in enumerate(names):
            set_address(kind, ctypes.cast(getattr(L, name), ctypes.c_void_p).value)
    for op, name in enumerate(("append", "read", "attention", "weights", "evict")):
        for fmt, entry in enumerate(_KV_FORMATS):
            binding.set_kv(op, fmt, ctypes.cast(getattr(L, f"torq_{entry}_kv_{name}"), ctypes.c_void_p).value)
    binding.set_kv(5, 0, ctypes.cast(L.torq_kv_attention_workspace_bytes, ctypes.c_void_p).value)
    _binding_module = binding
    return binding


def _layer_ctypes(kind, X, R, R_intra, Wq, Ws, Y, workspace, dbg_codes, dbg_scales, stream, x_scale=None, w_scale=None):
    for t, dtype, optional in ((X, torch.bfloat16, False), (R, torch.bfloat16, True), (R_intra, torch.bfloat16, True),
                               (Wq, torch.uint8, False), (Ws, torch.uint8, False), (Y, None, False), (workspace, None, False),
                               (dbg_codes, torch.uint8, True), (dbg_scales, torch.uint8, True)):
        if t is None and optional:
            continue
        if not (isinstance(t, torch.Tensor) and (dtype is None or t.dtype is dtype) and t.is_cuda and t.is_contiguous()):
            return -1
    if X.dim() != 2 or Wq.dim() < 1 or Y.dtype not in (torch.float32, torch.bfloat16) or Y.numel() < X.shape[0] * Wq.shape[0]:
        return -1
    M, d = X.shape
    rest = (M, d, Wq.shape[0], _ptr(Y), TORQ_F32 if Y.dtype == torch.float32 else TORQ_BF16, _ptr(workspace), workspace.numel(),
            _ptr(dbg_codes), _ptr(dbg_scales), _stream() if stream is None else stream)
    f = getattr(lib(), _LAYER_ENTRIES[kind])
    if kind == _NVFP4:
        return f(_ptr(X), _ptr(R), _ptr(R_intra), x_scale, _ptr(Wq), _ptr(Ws), w_scale, *rest)
    return f(_ptr(X), _ptr(R), _ptr(R_intra), _ptr(Wq), _ptr(Ws), *rest)


def _handle(stream):
    return None if stream is None else stream.cuda_stream


# The marshalling below is paid on every call, and a layer of a few tokens takes the GPU 13 us: addresses and
# streams therefore go to ctypes as plain integers (the argument types are declared, so it converts them itself),
# and the current stream is read as the raw handle (0.2 us; building a torch.cuda.Stream object for it took 3.6).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _check(t, dtype, name):
    if t is not None and not (t.dtype is dtype and t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{name}: expected a contiguous CUDA tensor of {dtype}, got {t.dtype} on {t.device}")


def _check_result(Y, M, N):
    """Y is written densely as float32 or bfloat16: anything else would get other bytes than its own, or bytes beside it."""
    if not (Y.dtype in (torch.float32, torch.bfloat16) and Y.is_cuda and Y.is_contiguous()):
        raise ValueError(f"Y: expected a contiguous CUDA tensor of float32 or bfloat16, got {Y.dtype} on {Y.device}")
    if Y.numel() < M * N:
        raise ValueError(f"Y: expected room for {M} x {N} values, got {tuple(Y.shape)}")


def _refuse(where, bf16, u8, Y, workspace):
    """Says what is wrong with the operands that the native binding did not take; nothing was launched."""
    X, Wq = bf16[0][1], u8[0][1]
    M, d = X.shape
    for n, t in bf16:
        _check(t, torch.bfloat16, n)
    for n, t in u8:
        _check(t, torch.uint8, n)
    _check_result(Y, M, Wq.shape[0])
    _check(workspace, workspace.dtype, "workspace")
    raise ValueError(f"{where}: an operand is not a plain CUDA tensor")


def _raise(code, where):
    if code != 0:
        raise TorqError(code, where)


def torq_scales_bytes(rows: int, k: int) -> int:
    return lib().torq_scales_bytes(rows, k)


def torq_scale_offset(row: int, kblock: int, k: int) -> int:
    return lib().torq_scale_offset(row, kblock, k)


def torq_workspace_bytes(M: int, d: int, N: int) -> int:
    return lib().torq_workspace_bytes(M, d, N)


def torq_pair_tile_list(rows: int, cols: int, pairs: int = 74):
    """[(row_tile, first_column, width), ...] in dealing order (host helper, no device work)."""
    n = lib().torq_pair_tile_list(rows, cols, pairs, None, 0)
    if n < 0:
        raise ValueError("torq_pair_tile_list: rows, cols and pairs must be positive")
    buf = (ctypes.c_int32 * (3 * n))()
    lib().torq_pair_tile_list(rows, cols, pairs, buf, n)
    return [(buf[3 * i], buf[3 * i + 1], buf[3 * i + 2]) for i in range(n)]


def torq_gemm_tile_list(M: int, N: int, w_row_bytes: int, pairs: int = 74):
    """The same for a GEMM, in its order (w_row_bytes: K / 2, MXINT4 K)."""
    n = lib().torq_gemm_tile_list(M, N, w_row_bytes, pairs, None, 0)
    if n < 0:
        raise ValueError("torq_gemm_tile_list: M, N, w_row_bytes and pairs must be positive")
    buf = (ctypes.c_int32 * (3 * n))()
    lib().torq_gemm_tile_list(M, N, w_row_bytes, pairs, buf, n)
    return [(buf[3 * i], buf[3 * i + 1], buf[3 * i + 2]) for i in range(n)]


def torq_launch_count() -> int:
    return lib().torq_launch_count()


def torq_last_device_error(stream=None) -> int:
    return lib().torq_last_device_error(_stream(stream))


def torq_quantize_mxfp4(Z, out_codes=None, out_scales=None, stream=None):
    """Z [M,d] float32 or bfloat16 -> (codes [M,d/2] uint8, tiled scale bytes uint8)."""
    M, d = Z.shape
    dt = TORQ_F32 if Z.dtype == torch.float32 else TORQ_BF16
    _check(Z, torch.float32 if dt == TORQ_F32 else torch.bfloat16, "Z")
    if out_codes is None:
        out_codes = torch.empty((M, d // 2), dtype=torch.uint8, device=Z.device)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=Z.device)
    _raise(lib().torq_quantize_mxfp4(_ptr(Z), dt, M, d, _ptr(out_codes), _ptr(out_scales), _stream(stream)),
           "torq_quantize_mxfp4")
    return out_codes, out_scales


def torq_rotate_quantize(X, R_inter, R_intra, out_codes=None, out_scales=None, stream=None):
    """X [M,d] bf16, R_inter [d,d] bf16 or None, R_intra [d/32,32,32] bf16 or None."""
    M, d = X.shape
    for t, n in ((X, "X"), (R_inter, "R_inter"), (R_intra, "R_intra")):
        _check(t, torch.bfloat16, n)
    if out_codes is None:
        out_codes = torch.empty((M, d // 2), dtype=torch.uint8, device=X.device)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
    _raise(lib().torq_rotate_quantize(_ptr(X), _ptr(R_inter), _ptr(R_intra), M, d, _ptr(out_codes),
                                      _ptr(out_scales), _stream(stream)), "torq_rotate_quantize")
    return out_codes, out_scales


def torq_rotate_quantize_structured(X, R_B, R_intra, out_codes=None, out_scales=None, stream=None):
    """X [M,d] bf16, R_B [d/32,d/32] bf16 (mixes the blocks of a token), R_intra [32,32] bf16 or None
    (shared by all blocks): the rotation in the structure the paper gives it."""
    M, d = X.shape
    for t, n in ((X, "X"), (R_B, "R_B"), (R_intra, "R_intra")):
        _check(t, torch.bfloat16, n)
    if out_codes is None:
        out_codes = torch.empty((M, d // 2), dtype=torch.uint8, device=X.device)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
    _raise(lib().torq_rotate_quantize_structured(_ptr(X), _ptr(R_B), _ptr(R_intra), M, d, _ptr(out_codes),
                                                 _ptr(out_scales), _stream(stream)), "torq_rotate_quantize_structured")
    return out_codes, out_scales


def torq_mxfp4_gemm(Aq, As, Wq, Ws, out_dtype=torch.bfloat16, Y=None, stream=None):
    """Aq [M,K/2], Wq [N,K/2] uint8 codes; As, Ws tiled scale bytes -> Y [M,N]."""
    M, K2 = Aq.shape
    N = Wq.shape[0]
    for t, n in ((Aq, "Aq"), (As, "As"), (Wq, "Wq"), (Ws, "Ws")):
        _check(t, torch.uint8, n)
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype, device=Aq.device)
    _check_result(Y, M, N)
    dt = TORQ_F32 if Y.dtype == torch.float32 else TORQ_BF16
    _raise(lib().torq_mxfp4_gemm(_ptr(Aq), _ptr(As), _ptr(Wq), _ptr(Ws), M, N, 2 * K2, _ptr(Y), dt,
                                 _stream(stream)), "torq_mxfp4_gemm")
    return Y


def torq_rotated_linear(X, R_inter, R_intra, Wq, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None,
                        dbg_codes=None, dbg_scales=None, stream=None):
    """Rotate, quantize and multiply in one call.  Returns Y [M,N]."""
    if Y is None:
        Y = torch.empty((X.shape[0], Wq.shape[0]), dtype=out_dtype, device=X.device)
    if workspace is None:
        M, d = X.shape
        workspace = torch.empty(torq_workspace_bytes(M, d, Wq.shape[0]), dtype=torch.uint8, device=X.device)
    rc = _layer(_MXFP4, X, R_inter, R_intra, Wq, Ws, Y, workspace, dbg_codes, dbg_scales, _handle(stream))
    if rc == 0:
        return Y
    if rc > 0:
        raise TorqError(rc, "torq_rotated_linear")
    _refuse("torq_rotated_linear", (("X", X), ("R_inter", R_inter), ("R_intra", R_intra)),
            (("Wq", Wq), ("Ws", Ws), ("dbg_codes", dbg_codes), ("dbg_scales", dbg_scales)), Y, workspace)


def torq_rotated_linear_structured(X, R_B, R_intra, Wq, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None,
                                   dbg_codes=None, dbg_scales=None, stream=None):
    """The whole layer with the rotation in the paper's structure (R_B [d/32,d/32], shared R_intra [32,32])."""
    if Y is None:
        Y = torch.empty((X.shape[0], Wq.shape[0]), dtype=out_dtype, device=X.device)
    if workspace is None:
        M, d = X.shape
        workspace = torch.empty(torq_workspace_bytes(M, d, Wq.shape[0]), dtype=torch.uint8, device=X.device)
    rc = _layer(_STRUCTURED, X, R_B, R_intra, Wq, Ws, Y, workspace, dbg_codes, dbg_scales, _handle(stream))
    if rc == 0:
        return Y
    if rc > 0:
        raise TorqError(rc, "torq_rotated_linear_structured")
    _refuse("torq_rotated_linear_structured", (("X", X), ("R_B", R_B), ("R_intra", R_intra)),
            (("Wq", Wq), ("Ws", Ws), ("dbg_codes", dbg_codes), ("dbg_scales", dbg_scales)), Y, workspace)


TORQ_STATIC_WORKSPACE_BYTES = 16 << 20


def torq_rotated_linear_static(X, R_inter, R_intra, Wq, Ws, Y, stream=None):
    """The whole layer for callers that cannot allocate device memory (a plug-in that only gets
    input and output pointers, a server whose memory is already committed to other pools, a
    decode loop that cannot afford the synchronisation an allocation implies).  The scratch for
    the quantized activations is a fixed array inside the library, TORQ_STATIC_WORKSPACE_BYTES
    long, shared by every call on the device; Y must be passed in, and this wrapper creates no
    tensor either.  Raises TorqError(TORQ_ERR_WORKSPACE) when the problem needs more scratch than
    the array holds.  Calls that may overlap on the GPU race on the array: keep them in one
    stream.  Make the first call on a device during start-up (it looks up the array's address)."""
    M, d = X.shape
    N = Wq.shape[0]
    for t, n in ((X, "X"), (R_inter, "R_inter"), (R_intra, "R_intra")):
        _check(t, torch.bfloat16, n)
    for t, n in ((Wq, "Wq"), (Ws, "Ws")):
        _check(t, torch.uint8, n)
    _check_result(Y, M, N)
    dt = TORQ_F32 if Y.dtype == torch.float32 else TORQ_BF16
    _raise(lib().torq_rotated_linear_static(_ptr(X), _ptr(R_inter), _ptr(R_intra), _ptr(Wq), _ptr(Ws), M, d, N,
                                            _ptr(Y), dt, _stream(stream)), "torq_rotated_linear_static")
    return Y


def torq_probe_fp4_peak(groups: int = 40000, stream=None) -> float:
    """Issue-bound rate (TFLOP/s) of the block-scaled FP4 tensor-core instruction on this device."""
    out = ctypes.c_double(0.0)
    _raise(lib().torq_probe_fp4_peak(groups, ctypes.byref(out), _stream(stream)), "torq_probe_fp4_peak")
    return out.value


def torq_selftest_wait_timeout(limit_ns: int = 1_000_000, stream=None):
    """Runs the give-up path of the bounded device waits once, harmlessly (see torq.h).  Returns a
    device int64 tensor [gave_up, left_through_abort_flag, waited_ns]."""
    out = torch.zeros(4, dtype=torch.int64, device="cuda")
    _raise(lib().torq_selftest_wait_timeout(int(limit_ns), _ptr(out), _stream(stream)), "torq_selftest_wait_timeout")
    return out[:3]


def torq_swizzle_scales(linear, k: int, out=None, stream=None):
    rows = linear.shape[0]
    _check(linear, torch.uint8, "linear")
    if out is None:
        out = torch.empty(torq_scales_bytes(rows, k), dtype=torch.uint8, device=linear.device)
    _raise(lib().torq_swizzle_scales(_ptr(linear), rows, k, _ptr(out), _stream(stream)), "torq_swizzle_scales")
    return out


def torq_merge_rotations(R_inter, R_intra, out=None, stream=None):
    d = R_inter.shape[0]
    _check(R_inter, torch.bfloat16, "R_inter")
    _check(R_intra, torch.bfloat16, "R_intra")
    if out is None:
        out = torch.empty((d, d), dtype=torch.float32, device=R_inter.device)
    _raise(lib().torq_merge_rotations(_ptr(R_inter), _ptr(R_intra), d, _ptr(out), _stream(stream)),
           "torq_merge_rotations")
    return out


def torq_merge_rotations_bf16(R_inter, R_intra, out=None, stream=None):
    """R~ = R_inter blockdiag(R_intra) rounded once to bfloat16: the operand of the one-GEMM form of the rotation."""
    d = R_inter.shape[0]
    _check(R_inter, torch.bfloat16, "R_inter")
    _check(R_intra, torch.bfloat16, "R_intra")
    if out is None:
        out = torch.empty((d, d), dtype=torch.bfloat16, device=R_inter.device)
    _raise(lib().torq_merge_rotations_bf16(_ptr(R_inter), _ptr(R_intra), d, _ptr(out), _stream(stream)),
           "torq_merge_rotations_bf16")
    return out


def torq_prepare_weights_workspace_bytes(d: int, N: int) -> int:
    return int(lib().torq_prepare_weights_workspace_bytes(d, N))


def _prep_args(R_inter, R_intra, W, workspace):
    _check(W, torch.float32, "W")
    _check(R_inter, torch.bfloat16, "R_inter")
    _check(R_intra, torch.bfloat16, "R_intra")
    d, N = W.shape
    if workspace is None:
        workspace = torch.empty(torq_prepare_weights_workspace_bytes(d, N), dtype=torch.uint8, device=W.device)
    return d, N, workspace


def torq_prepare_weights(R_inter, R_intra, W, workspace=None, stream=None):
    """Offline weight side of the layer: W [d,N] float32 -> (Wq [N,d/2], Ws tiled), W' = R~^T W quantized
    to MXFP4 along K, all of it by the library's kernels."""
    d, N, workspace = _prep_args(R_inter, R_intra, W, workspace)
    Wq = torch.empty((N, d // 2), dtype=torch.uint8, device=W.device)
    Ws = torch.empty(torq_scales_bytes(N, d), dtype=torch.uint8, device=W.device)
    _raise(lib().torq_prepare_weights(_ptr(W), _ptr(R_inter), _ptr(R_intra), d, N, _ptr(Wq), _ptr(Ws),
                                      _ptr(workspace), workspace.numel(), _stream(stream)), "torq_prepare_weights")
    return Wq, Ws


prepare_weights = torq_prepare_weights


# ---- NVFP4 variant (16-element blocks, E4M3 block scales, float32 tensor scale) -----------------------
def torq_nvfp4_scales_bytes(rows: int, k: int) -> int:
    return lib().torq_nvfp4_scales_bytes(rows, k)


def torq_nvfp4_workspace_bytes(M: int, d: int, N: int) -> int:
    return lib().torq_nvfp4_workspace_bytes(M, d, N)


def torq_expand_intra16(R_intra16, out=None, stream=None):
    """[d/16,16,16] bf16 -> the 32-wide block-diagonal form [d/32,32,32] the rotation kernels take."""
    _check(R_intra16, torch.bfloat16, "R_intra16")
    d = R_intra16.shape[0] * 16
    if out is None:
        out = torch.empty((d // 32, 32, 32), dtype=torch.bfloat16, device=R_intra16.device)
    _raise(lib().torq_expand_intra16(_ptr(R_intra16), d, _ptr(out), _stream(stream)), "torq_expand_intra16")
    return out


def torq_quantize_nvfp4(Z, tensor_scale: float, out_codes=None, out_scales=None, stream=None):
    """Z [M,d] float32 or bfloat16 -> (codes [M,d/2] uint8, tiled E4M3 scale bytes uint8)."""
    M, d = Z.shape
    dt = TORQ_F32 if Z.dtype == torch.float32 else TORQ_BF16
    _check(Z, torch.float32 if dt == TORQ_F32 else torch.bfloat16, "Z")
    if out_codes is None:
        out_codes = torch.empty((M, d // 2), dtype=torch.uint8, device=Z.device)
    if out_scales is None:
        out_scales = torch.empty(torq_nvfp4_scales_bytes(M, d), dtype=torch.uint8, device=Z.device)
    _raise(lib().torq_quantize_nvfp4(_ptr(Z), dt, M, d, tensor_scale, _ptr(out_codes), _ptr(out_scales),
                                     _stream(stream)), "torq_quantize_nvfp4")
    return out_codes, out_scales


def torq_rotate_quantize_nvfp4(X, R_inter, R_intra32, tensor_scale: float, out_codes=None, out_scales=None,
                               stream=None):
    """X [M,d] bf16, R_inter [d,d] bf16, R_intra32 [d/32,32,32] bf16 or None (see torq_expand_intra16)."""
    M, d = X.shape
    for t, n in ((X, "X"), (R_inter, "R_inter"), (R_intra32, "R_intra32")):
        _check(t, torch.bfloat16, n)
    if out_codes is None:
        out_codes = torch.empty((M, d // 2), dtype=torch.uint8, device=X.device)
    if out_scales is None:
        out_scales = torch.empty(torq_nvfp4_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
    _raise(lib().torq_rotate_quantize_nvfp4(_ptr(X), _ptr(R_inter), _ptr(R_intra32), M, d, tensor_scale,
                                            _ptr(out_codes), _ptr(out_scales), _stream(stream)),
           "torq_rotate_quantize_nvfp4")
    return out_codes, out_scales


def torq_nvfp4_gemm(Aq, As, a_tensor_scale: float, Wq, Ws, w_tensor_scale: float, out_dtype=torch.bfloat16, Y=None,
                    stream=None):
    """Aq [M,K/2], Wq [N,K/2] uint8 codes; As, Ws tiled E4M3 scale bytes -> Y [M,N]."""
    M, K2 = Aq.shape
    N = Wq.shape[0]
    for t, n in ((Aq, "Aq"), (As, "As"), (Wq, "Wq"), (Ws, "Ws")):
        _check(t, torch.uint8, n)
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype, device=Aq.device)
    _check_result(Y, M, N)
    dt = TORQ_F32 if Y.dtype == torch.float32 else TORQ_BF16
    _raise(lib().torq_nvfp4_gemm(_ptr(Aq), _ptr(As), a_tensor_scale, _ptr(Wq), _ptr(Ws), w_tensor_scale, M, N,
                                 2 * K2, _ptr(Y), dt, _stream(stream)), "torq_nvfp4_gemm")
    return Y


def torq_rotated_linear_nvfp4(X, R_inter, R_intra32, x_tensor_scale: float, Wq, Ws, w_tensor_scale: float,
                              out_dtype=torch.bfloat16, Y=None, workspace=None, dbg_codes=None, dbg_scales=None,
                              stream=None):
    """Rotate, quantize to NVFP4 and multiply in one call.  Returns Y [M,N]."""
    if Y is None:
        Y = torch.empty((X.shape[0], Wq.shape[0]), dtype=out_dtype, device=X.device)
    if workspace is None:
        M, d = X.shape
        workspace = torch.empty(torq_nvfp4_workspace_bytes(M, d, Wq.shape[0]), dtype=torch.uint8, device=X.device)
    rc = _layer(_NVFP4, X, R_inter, R_intra32, Wq, Ws, Y, workspace, dbg_codes, dbg_scales, _handle(stream), x_tensor_scale, w_tensor_scale)
    if rc == 0:
        return Y
    if rc > 0:
        raise TorqError(rc, "torq_rotated_linear_nvfp4")
    _refuse("torq_rotated_linear_nvfp4", (("X", X), ("R_inter", R_inter), ("R_intra32", R_intra32)),
            (("Wq", Wq), ("Ws", Ws), ("dbg_codes", dbg_codes), ("dbg_scales", dbg_scales)), Y, workspace)


def torq_prepare_weights_nvfp4(R_inter, R_intra32, W, workspace=None, stream=None):
    """Offline weight side in NVFP4: returns (Wq [N,d/2], Ws tiled, tensor_scale = max|W'| / (6 * 448)).
    Synchronises the stream once (the tensor scale comes back to the host)."""
    d, N, workspace = _prep_args(R_inter, R_intra32, W, workspace)
    Wq = torch.empty((N, d // 2), dtype=torch.uint8, device=W.device)
    Ws = torch.empty(torq_nvfp4_scales_bytes(N, d), dtype=torch.uint8, device=W.device)
    ts = ctypes.c_float(0.0)
    _raise(lib().torq_prepare_weights_nvfp4(_ptr(W), _ptr(R_inter), _ptr(R_intra32), d, N, _ptr(Wq), _ptr(Ws),
                                            ctypes.byref(ts), _ptr(workspace), workspace.numel(), _stream(stream)),
           "torq_prepare_weights_nvfp4")
    return Wq, Ws, ts.value


prepare_weights_nvfp4 = torq_prepare_weights_nvfp4


# ---- MXINT4 variant (format study of Section 6) ---------------------------------------------------------
def torq_mxint4_workspace_bytes(M: int, d: int, N: int) -> int:
    return int(lib().torq_mxint4_workspace_bytes(M, d, N))


def torq_quantize_mxint4(Z, packed: bool = False, out_codes=None, out_scales=None, stream=None):
    """Z [M,d] float32 or bfloat16 -> (codes, tiled E8M0 scale bytes).  packed: [M,d/2] two's-complement
    nibbles (stored form); otherwise [M,d] E4M3 bytes whose values are the integer codes (operand form)."""
    M, d = Z.shape
    dt = TORQ_F32 if Z.dtype == torch.float32 else TORQ_BF16
    _check(Z, torch.float32 if dt == TORQ_F32 else torch.bfloat16, "Z")
    if out_codes is None:
        out_codes = torch.empty((M, d // 2 if packed else d), dtype=torch.uint8, device=Z.device)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=Z.device)
    _check(out_codes, torch.uint8, "out_codes")
    _check(out_scales, torch.uint8, "out_scales")
    _raise(lib().torq_quantize_mxint4(_ptr(Z), dt, M, d, 1 if packed else 0, _ptr(out_codes), _ptr(out_scales),
                                      _stream(stream)), "torq_quantize_mxint4")
    return out_codes, out_scales


def torq_mxint4_expand(packed, out=None, stream=None):
    """Stored form [rows,k/2] -> operand form [rows,k]."""
    _check(packed, torch.uint8, "packed")
    rows, k2 = packed.shape
    if out is None:
        out = torch.empty((rows, 2 * k2), dtype=torch.uint8, device=packed.device)
    _check(out, torch.uint8, "out")
    _raise(lib().torq_mxint4_expand(_ptr(packed), rows, 2 * k2, _ptr(out), _stream(stream)), "torq_mxint4_expand")
    return out


def torq_rotate_quantize_mxint4(X, R_inter, R_intra, out_bytes=None, out_scales=None, stream=None):
    """X [M,d] bf16, R_inter [d,d] bf16, R_intra [d/32,32,32] bf16 or None -> (operand bytes [M,d], scales)."""
    M, d = X.shape
    for t, n in ((X, "X"), (R_inter, "R_inter"), (R_intra, "R_intra")):
        _check(t, torch.bfloat16, n)
    if out_bytes is None:
        out_bytes = torch.empty((M, d), dtype=torch.uint8, device=X.device)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
    _raise(lib().torq_rotate_quantize_mxint4(_ptr(X), _ptr(R_inter), _ptr(R_intra), M, d, _ptr(out_bytes),
                                             _ptr(out_scales), _stream(stream)), "torq_rotate_quantize_mxint4")
    return out_bytes, out_scales


def torq_rotate_quantize_structured_mxint4(X, R_B, R_intra, out_bytes=None, out_scales=None, stream=None):
    """The structured rotation (R_B [d/32,d/32], shared R_intra [32,32] or None) followed by the MXINT4 quantizer."""
    M, d = X.shape
    for t, n in ((X, "X"), (R_B, "R_B"), (R_intra, "R_intra")):
        _check(t, torch.bfloat16, n)
    if out_bytes is None:
        out_bytes = torch.empty((M, d), dtype=torch.uint8, device=X.device)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
    _raise(lib().torq_rotate_quantize_structured_mxint4(_ptr(X), _ptr(R_B), _ptr(R_intra), M, d, _ptr(out_bytes),
                                                        _ptr(out_scales), _stream(stream)),
           "torq_rotate_quantize_structured_mxint4")
    return out_bytes, out_scales


def torq_mxint4_gemm(A8, As, W8, Ws, out_dtype=torch.bfloat16, Y=None, stream=None):
    """A8 [M,K], W8 [N,K] operand bytes; As, Ws tiled E8M0 scale bytes -> Y [M,N]."""
    M, K = A8.shape
    N = W8.shape[0]
    for t, n in ((A8, "A8"), (As, "As"), (W8, "W8"), (Ws, "Ws")):
        _check(t, torch.uint8, n)
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype, device=A8.device)
    _check_result(Y, M, N)
    dt = TORQ_F32 if Y.dtype == torch.float32 else TORQ_BF16
    _raise(lib().torq_mxint4_gemm(_ptr(A8), _ptr(As), _ptr(W8), _ptr(Ws), M, N, K, _ptr(Y), dt, _stream(stream)),
           "torq_mxint4_gemm")
    return Y


def torq_rotated_linear_mxint4(X, R_inter, R_intra, W8, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None,
                               dbg_bytes=None, dbg_scales=None, stream=None):
    """Rotate, quantize to MXINT4 and multiply in one call.  Returns Y [M,N]."""
    if Y is None:
        Y = torch.empty((X.shape[0], W8.shape[0]), dtype=out_dtype, device=X.device)
    if workspace is None:
        M, d = X.shape
        workspace = torch.empty(torq_mxint4_workspace_bytes(M, d, W8.shape[0]), dtype=torch.uint8, device=X.device)
    rc = _layer(_MXINT4, X, R_inter, R_intra, W8, Ws, Y, workspace, dbg_bytes, dbg_scales, _handle(stream))
    if rc == 0:
        return Y
    if rc > 0:
        raise TorqError(rc, "torq_rotated_linear_mxint4")
    _refuse("torq_rotated_linear_mxint4", (("X", X), ("R_inter", R_inter), ("R_intra", R_intra)),
            (("W8", W8), ("Ws", Ws), ("dbg_bytes", dbg_bytes), ("dbg_scales", dbg_scales)), Y, workspace)


def torq_prepare_weights_mxint4(R_inter, R_intra, W, workspace=None, stream=None):
    """Offline weight side in MXINT4: returns (stored form [N,d/2], operand form [N,d], tiled scales)."""
    d, N, workspace = _prep_args(R_inter, R_intra, W, workspace)
    Wn = torch.empty((N, d // 2), dtype=torch.uint8, device=W.device)
    W8 = torch.empty((N, d), dtype=torch.uint8, device=W.device)
    Ws = torch.empty(torq_scales_bytes(N, d), dtype=torch.uint8, device=W.device)
    _raise(lib().torq_prepare_weights_mxint4(_ptr(W), _ptr(R_inter), _ptr(R_intra), d, N, _ptr(Wn), _ptr(W8), _ptr(Ws),
                                             _ptr(workspace), workspace.numel(), _stream(stream)),
           "torq_prepare_weights_mxint4")
    return Wn, W8, Ws


prepare_weights_mxint4 = torq_prepare_weights_mxint4


# ---- operators around the layer: norm, products of few tokens, gated projections -----------------------
def _operand(t, dtypes, name, shape=None, at_least=None):
    """A contiguous CUDA tensor of the current device, of one of `dtypes`, of that shape, or with room for so many elements."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or not t.is_cuda or not t.is_contiguous():
        what = f"{t.dtype} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name}: expected a contiguous CUDA tensor of {' or '.join(str(d) for d in dtypes)}, got {what}")
    if t.device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: is on {t.device}, the call goes to the current device, cuda:{torch._C._cuda_getDevice()}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected the shape {tuple(shape)}, got {tuple(t.shape)}")
    if at_least is not None and t.numel() < at_least:
        raise ValueError(f"{name}: expected room for {at_least} elements, got {tuple(t.shape)}")


def _used_by(stream, *tensors):
    """Tensors made for a call on another stream than the current one: the allocator has to know that it uses them."""
    if stream is not None:
        for t in tensors:
            t.record_stream(stream)


_FLOATS = (torch.float32, torch.bfloat16)
_BYTES = (torch.uint8,)


def _dtype_code(t):
    return TORQ_F32 if t.dtype is torch.float32 else TORQ_BF16


def _norm_operands(X, weight, residual, residual_out, stream):
    _operand(X, _FLOATS, "X")
    if X.dim() != 2:
        raise ValueError(f"X: expected two dimensions, got {tuple(X.shape)}")
    M, d = X.shape
    _operand(weight, (torch.bfloat16,), "weight", (d,))
    if residual is None:
        if residual_out is not None:
            raise ValueError("residual_out without a residual")
        return M, d, None, TORQ_BF16
    _operand(residual, _FLOATS, "residual", (M, d))
    if residual_out is None:
        residual_out = torch.empty_like(residual)
        _used_by(stream, residual_out)
    _operand(residual_out, (residual.dtype,), "residual_out", (M, d))
    return M, d, residual_out, _dtype_code(residual)


def _product_native(*args):                      # until the first call has put the native function here
    global _product_native
    binding = _native_binding()
    _product_native = binding.product if binding else lambda *args: -1
    return _product_native(*args)


def _norm_native(*args):
    global _norm_native
    binding = _native_binding()
    _norm_native = binding.norm if binding else lambda *args: -1
    return _norm_native(*args)


def _norm(mx, X, weight, residual, eps, out, out_scales, residual_out, stream):
    """The norm through ctypes, with reasons for what it refuses: the tuple of results."""
    M, d, h, r_dtype = _norm_operands(X, weight, residual, residual_out, stream)
    if out is None:
        out = torch.empty((M, d), dtype=torch.uint8 if mx else torch.bfloat16, device=X.device)
        _used_by(stream, out)
    _operand(out, _BYTES if mx else (torch.bfloat16,), "out_bytes" if mx else "out", (M, d))
    args = (_ptr(X), _dtype_code(X), _ptr(residual), _ptr(h), r_dtype, _ptr(weight), eps, M, d, _ptr(out))
    if not mx:
        _raise(lib().torq_add_rmsnorm(*args, _stream(stream)), "torq_add_rmsnorm")
        return (out,) if h is None else (out, h)
    if out_scales is None:
        out_scales = torch.empty(torq_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
        _used_by(stream, out_scales)
    _operand(out_scales, _BYTES, "out_scales", at_least=torq_scales_bytes(M, d))
    _raise(lib().torq_add_rmsnorm_mxfp8(*args, _ptr(out_scales), _stream(stream)), "torq_add_rmsnorm_mxfp8")
    return (out, out_scales) if h is None else (out, out_scales, h)


def torq_add_rmsnorm(X, weight, residual=None, eps: float = 1e-6, out=None, residual_out=None, stream=None):
    """h = X + residual; y = h / sqrt(mean(h^2) + eps) * weight.  X, residual [M,d] float32 or bfloat16, weight [d] bf16.
    Returns y [M,d] bf16, or (y, h) with a residual, h in its type (residual_out=residual: in place)."""
    r = _norm_native(False, X, weight, residual, eps, out, None, residual_out, _handle(stream))
    if r.__class__ is int:
        if r > 0:
            raise TorqError(r, "torq_add_rmsnorm")
        r = _norm(False, X, weight, residual, eps, out, None, residual_out, stream)
    return r[0] if residual is None else r


def torq_add_rmsnorm_mxfp8(X, weight, residual=None, eps: float = 1e-6, out_bytes=None, out_scales=None, residual_out=None,
                           stream=None):
    """torq_add_rmsnorm with y as MXFP8: (E4M3 bytes [M,d] uint8, tiled E8M0 scale bytes[, h]), the A operand of
    torq_mxint4_gemm and torq_mxint4_gated_gemm."""
    r = _norm_native(True, X, weight, residual, eps, out_bytes, out_scales, residual_out, _handle(stream))
    if r.__class__ is int:
        if r > 0:
            raise TorqError(r, "torq_add_rmsnorm_mxfp8")
        r = _norm(True, X, weight, residual, eps, out_bytes, out_scales, residual_out, stream)
    return r


_IN_BF16 = object()


def torq_matvec_workspace_bytes(M: int, N: int, K: int) -> int:
    return lib().torq_matvec_workspace_bytes(M, N, K)


def _product(kind, A, As, Wq, Ws, out_dtype, Y, stream, a_scale=0.0, w_scale=0.0, workspace=None):
    """Y = A W^T of one format and kind (a number in _OPERATORS).  As _IN_BF16: A is bf16 [M,K]; else codes, as Wq's are."""
    if Y is not None or out_dtype in _FLOATS:
        r = _product_native(kind, A, As, Wq, Ws, Y, out_dtype is torch.float32, _handle(stream), a_scale, w_scale, workspace)
        if r.__class__ is not int:
            return r
        if r > 0:
            raise TorqError(r, _OPERATORS[kind])
    # through ctypes, with reasons for what it refuses
    name, per_byte, gated = _OPERATORS[kind], 1 if kind == 8 else 2, kind >= 3
    scales = (a_scale, w_scale) if kind % 3 == 1 else ()
    bf16 = As is _IN_BF16
    _operand(A, (torch.bfloat16,) if bf16 else _BYTES, "X" if bf16 else "A")
    _operand(Wq, _BYTES, "W")
    if A.dim() != 2 or Wq.dim() != 2:
        raise ValueError(f"{name}: expected matrices, got {tuple(A.shape)} and {tuple(Wq.shape)}")
    M, rows, K = A.shape[0], Wq.shape[0], Wq.shape[1] * per_byte
    if A.shape[1] * (1 if bf16 else per_byte) != K:
        raise ValueError(f"{name}: {tuple(A.shape)} and {tuple(Wq.shape)} have different K")
    scales_bytes = torq_nvfp4_scales_bytes if scales else torq_scales_bytes
    _operand(Ws, _BYTES, "Ws", at_least=scales_bytes(rows, K))
    if not bf16:
        _operand(As, _BYTES, "As", at_least=scales_bytes(M, K))
    if gated and rows % 2:
        raise ValueError(f"{name}: W has gate and up rows, got an odd number of them")
    N = rows // 2 if gated else rows
    if Y is None:
        if out_dtype not in _FLOATS:
            raise ValueError(f"{name}: expected an out_dtype of {' or '.join(str(d) for d in _FLOATS)}, got {out_dtype}")
        Y = torch.empty((M, N), dtype=out_dtype, device=A.device)
        _used_by(stream, Y)
    _operand(Y, _FLOATS, "Y", (M, N))
    x = (_ptr(A),) if bf16 else (_ptr(A), _ptr(As), *scales[:1])
    scratch = ()
    if bf16:
        if workspace is None:
            workspace = torch.empty(torq_matvec_workspace_bytes(M, N, K), dtype=torch.uint8, device=A.device)
            _used_by(stream, workspace)
        _operand(workspace, (getattr(workspace, "dtype", "any type"),), "workspace")
        scratch = (_ptr(workspace), workspace.nbytes)
    _raise(getattr(lib(), name)(*x, _ptr(Wq), _ptr(Ws), *scales[-1:], M, N, K, _ptr(Y), _dtype_code(Y), *scratch, _stream(stream)), name)
    return Y


def torq_mxfp4_matvec(X, Wq, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None, stream=None):
    """X [M,K] bf16 (few tokens) times MXFP4 weights Wq [N,K/2], Ws tiled -> Y [M,N]."""
    return _product(0, X, _IN_BF16, Wq, Ws, out_dtype, Y, stream, workspace=workspace)


def torq_nvfp4_matvec(X, Wq, Ws, w_tensor_scale: float, out_dtype=torch.bfloat16, Y=None, workspace=None, stream=None):
    """X [M,K] bf16 (few tokens) times NVFP4 weights Wq [N,K/2], Ws tiled -> Y [M,N]."""
    return _product(1, X, _IN_BF16, Wq, Ws, out_dtype, Y, stream, w_scale=w_tensor_scale, workspace=workspace)


def torq_mxint4_matvec(X, Wn, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None, stream=None):
    """X [M,K] bf16 (few tokens) times MXINT4 weights in their stored form Wn [N,K/2], Ws tiled -> Y [M,N]."""
    return _product(2, X, _IN_BF16, Wn, Ws, out_dtype, Y, stream, workspace=workspace)


def torq_mxfp4_gated_matvec(X, Wq, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None, stream=None):
    """silu(X Wg^T) * (X Wu^T) of few tokens, X [M,K] bf16, Wq [2N,K/2] MXFP4 with the gate rows first -> Y [M,N]."""
    return _product(3, X, _IN_BF16, Wq, Ws, out_dtype, Y, stream, workspace=workspace)


def torq_nvfp4_gated_matvec(X, Wq, Ws, w_tensor_scale: float, out_dtype=torch.bfloat16, Y=None, workspace=None, stream=None):
    """The same with NVFP4 weights."""
    return _product(4, X, _IN_BF16, Wq, Ws, out_dtype, Y, stream, w_scale=w_tensor_scale, workspace=workspace)


def torq_mxint4_gated_matvec(X, Wn, Ws, out_dtype=torch.bfloat16, Y=None, workspace=None, stream=None):
    """The same with MXINT4 weights in their stored form."""
    return _product(5, X, _IN_BF16, Wn, Ws, out_dtype, Y, stream, workspace=workspace)


def torq_mxfp4_gated_gemm(Aq, As, Wq, Ws, out_dtype=torch.bfloat16, Y=None, stream=None):
    """silu(A Wg^T) * (A Wu^T): Aq [M,K/2], Wq [2N,K/2] MXFP4 codes with the gate rows first, As, Ws tiled -> Y [M,N]."""
    return _product(6, Aq, As, Wq, Ws, out_dtype, Y, stream)


def torq_nvfp4_gated_gemm(Aq, As, a_tensor_scale: float, Wq, Ws, w_tensor_scale: float, out_dtype=torch.bfloat16, Y=None,
                          stream=None):
    """The same on NVFP4 operands."""
    return _product(7, Aq, As, Wq, Ws, out_dtype, Y, stream, a_tensor_scale, w_tensor_scale)


def torq_mxint4_gated_gemm(A8, As, W8, Ws, out_dtype=torch.bfloat16, Y=None, stream=None):
    """The same on operand bytes: A8 [M,K] E4M3 with E8M0 scales (MXINT4 or torq_add_rmsnorm_mxfp8's), W8 [2N,K]."""
    return _product(8, A8, As, W8, Ws, out_dtype, Y, stream)


# ---- a key/value cache in 4 bits -----------------------------------------------------------------------
# pages [num_pages, kv_heads, bytes] uint8, table [batch, width], lengths [batch] and starts [batch + 1] int32; see torq_kv_cache in the
# header for the layout of a page and for what a call's rows are.
_INTS = (torch.int32,)


def torq_kv_page_bytes(fmt: str, page_tokens: int, head_dim: int) -> int:
    """Bytes of one head's page: the last dimension of pages.  fmt: "mxfp4", "nvfp4" or "mxint4"."""
    return int(lib().torq_kv_page_bytes(16 if fmt == "nvfp4" else 32, page_tokens, head_dim))


def torq_kv_attention_workspace_bytes(tokens: int, batch: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().torq_kv_attention_workspace_bytes(tokens, batch, heads, kv_heads, head_dim))


def _kv_rows(t, dtypes, name):
    """[tokens, heads, dim] with dense rows that may lie apart: the distance between rows."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or not t.is_cuda or t.dim() != 3:
        what = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name}: expected a CUDA tensor [tokens, heads, dim] of {' or '.join(str(d) for d in dtypes)}, got {what}")
    _here(t, name)
    tokens, heads, dim = t.shape
    if t.stride(2) != 1 and dim > 1 or t.stride(1) != dim and heads > 1 or t.stride(0) < heads * dim and tokens > 1:
        raise ValueError(f"{name}: the heads of a row have to lie one behind the other, got strides {t.stride()}")
    return t.stride(0) if tokens > 1 else heads * dim


def _here(t, name):
    if t.device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: is on {t.device}, the call goes to the current device, cuda:{torch._C._cuda_getDevice()}")


def _kv_cache(fmt, pages, table, lengths, dim, scales, starts, tokens):
    _operand(pages, _BYTES, "pages")
    _operand(table, _INTS, "table")
    if pages.dim() != 3 or table.dim() != 2:
        raise ValueError(f"expected pages [num_pages, kv_heads, bytes] and table [batch, width], got {tuple(pages.shape)} and {tuple(table.shape)}")
    batch = table.shape[0]
    _operand(lengths, _INTS, "lengths", (batch,))
    if starts is not None:
        _operand(starts, _INTS, "starts", (batch + 1,))
    elif tokens != batch:
        raise ValueError(f"{tokens} tokens of {batch} sequences: starts says which are whose")
    one = torq_kv_page_bytes(fmt, 1, dim)
    if dim not in (64, 128, 256) or pages.shape[2] % one:
        raise ValueError(f"pages: {pages.shape[2]} bytes of a head are no whole tokens of head dimension {dim}")
    return _KvCache(_ptr(pages), _ptr(table), _ptr(lengths), pages.shape[0], pages.shape[2] // one, pages.shape[1], dim, batch,
                    table.shape[1], *(scales or (1.0, 1.0)))


def _kv_scoring(scale, softcap, slopes, window, prefix, first, dim, heads, batch, tokens):
    if slopes is not None:
        _operand(slopes, (torch.float32,), "slopes", (heads,))
    if prefix is not None:
        _operand(prefix, _INTS, "prefix", (batch,))
    if first is not None:
        _operand(first, _INTS, "first", (tokens,))
    return _KvScoring(dim ** -0.5 if scale is None else scale, softcap, _ptr(slopes), window, _ptr(prefix), _ptr(first))


class _KvNative:
    """The native functions of the cache's calls, looked up at the first one; -1 where they cannot be had."""

    def __getattr__(self, name):
        binding = _native_binding()
        f = getattr(binding, name) if binding else lambda *args: -1
        setattr(self, name, f)
        return f


_kv_native = _KvNative()


def _kv_append(fmt, pages, table, lengths, K, V, scales, starts, stream):
    r = _kv_native.kv_append(_KV_FORMATS.index(fmt), pages, table, lengths, K, V, starts, *(scales or (1.0, 1.0)), _handle(stream))
    if r >= 0:
        return _raise(r, f"torq_{fmt}_kv_append")
    strides = _kv_rows(K, _FLOATS, "K"), _kv_rows(V, (getattr(K, "dtype", None),), "V")
    cache = _kv_cache(fmt, pages, table, lengths, K.shape[2], scales, starts, K.shape[0])
    if K.shape != V.shape or K.shape[1] != pages.shape[1]:
        raise ValueError(f"K and V: {tuple(K.shape)} and {tuple(V.shape)} do not fit {pages.shape[1]} heads")
    name = f"torq_{fmt}_kv_append"
    _raise(getattr(lib(), name)(cache, _ptr(K), _ptr(V), _dtype_code(K), *strides, _ptr(starts), K.shape[0], _stream(stream)), name)


def _kv_read(fmt, pages, table, lengths, head_dim, tokens, scales, starts, out_dtype, stream):
    if out_dtype in _FLOATS:
        r = _kv_native.kv_read(_KV_FORMATS.index(fmt), pages, table, lengths, head_dim, tokens, starts, *(scales or (1.0, 1.0)),
                               out_dtype is torch.float32, _handle(stream))
        if r.__class__ is not int:
            return r
        if r > 0:
            raise TorqError(r, f"torq_{fmt}_kv_read")
    cache = _kv_cache(fmt, pages, table, lengths, head_dim, scales, starts, tokens)
    name = f"torq_{fmt}_kv_read"
    if out_dtype not in _FLOATS:
        raise ValueError(f"{name}: expected an out_dtype of {' or '.join(str(d) for d in _FLOATS)}, got {out_dtype}")
    K, V = (torch.empty((tokens, pages.shape[1], head_dim), dtype=out_dtype, device=pages.device) for _ in range(2))
    _used_by(stream, K, V)
    _raise(getattr(lib(), name)(cache, _ptr(starts), tokens, _ptr(K), _ptr(V), _dtype_code(K), _stream(stream)), name)
    return K, V


def _kv_queries(fmt, pages, table, lengths, Q, scales, starts):
    stride = _kv_rows(Q, (torch.bfloat16,), "Q")
    tokens, heads, dim = Q.shape
    cache = _kv_cache(fmt, pages, table, lengths, dim, scales, starts, tokens)
    if not heads or not pages.shape[1] or heads % pages.shape[1]:
        raise ValueError(f"Q: {heads} heads do not share {pages.shape[1]} key/value heads evenly")
    return cache, stride, tokens, heads, dim


def _kv_attention(fmt, pages, table, lengths, Q, scales, starts, scale, softcap, slopes, window, prefix, first, out, return_lse, workspace,
                  stream):
    r = _kv_native.kv_attention(_KV_FORMATS.index(fmt), pages, table, lengths, Q, starts, *(scales or (1.0, 1.0)), scale, softcap, slopes, window,
                                prefix, first, out, return_lse, workspace, _handle(stream))
    if r.__class__ is not int:
        return r
    if r > 0:
        raise TorqError(r, f"torq_{fmt}_kv_attention")
    # through ctypes, with reasons for what it refuses
    cache, stride, tokens, heads, dim = _kv_queries(fmt, pages, table, lengths, Q, scales, starts)
    scoring = _kv_scoring(scale, softcap, slopes, window, prefix, first, dim, heads, cache.batch, tokens)
    if out is None:
        out = torch.empty((tokens, heads, dim), dtype=torch.bfloat16, device=Q.device)
        _used_by(stream, out)
    _operand(out, (torch.bfloat16,), "out", (tokens, heads, dim))
    lse = None
    if return_lse:
        lse = torch.empty((tokens, heads), dtype=torch.float32, device=Q.device)
        _used_by(stream, lse)
    if workspace is None:
        workspace = torch.empty(torq_kv_attention_workspace_bytes(tokens, cache.batch, heads, cache.kv_heads, dim), dtype=torch.uint8, device=Q.device)
        _used_by(stream, workspace)
    _operand(workspace, (getattr(workspace, "dtype", "any type"),), "workspace")
    name = f"torq_{fmt}_kv_attention"
    _raise(getattr(lib(), name)(cache, scoring, _ptr(Q), stride, heads, _ptr(starts), tokens, _ptr(out), _ptr(lse), _ptr(workspace),
                                workspace.nbytes, _stream(stream)), name)
    return (out, lse) if return_lse else out


def _kv_weights(fmt, pages, table, lengths, Q, lse, weights, scales, starts, scale, softcap, slopes, window, prefix, first, weights_out, stream):
    r = _kv_native.kv_weights(_KV_FORMATS.index(fmt), pages, table, lengths, Q, lse, weights, starts, scales[0] if scales else 1.0, scale, softcap, slopes,
                              window, prefix, first, weights_out, _handle(stream))
    if r >= 0:
        _raise(r, f"torq_{fmt}_kv_weights")
        return weights if weights_out is None else weights_out
    cache, stride, tokens, heads, dim = _kv_queries(fmt, pages, table, lengths, Q, scales, starts)
    scoring = _kv_scoring(scale, softcap, slopes, window, prefix, first, dim, heads, cache.batch, tokens)
    _operand(lse, (torch.float32,), "lse", (tokens, heads))
    shape = (cache.num_pages, cache.kv_heads, cache.page_tokens)
    _operand(weights, (torch.float32,), "weights", shape)
    if weights_out is None:
        weights_out = weights
    _operand(weights_out, (torch.float32,), "weights_out", shape)
    name = f"torq_{fmt}_kv_weights"
    _raise(getattr(lib(), name)(cache, scoring, _ptr(Q), stride, heads, _ptr(starts), tokens, _ptr(lse), _ptr(weights), _ptr(weights_out),
                                _stream(stream)), name)
    return weights_out


def _kv_evict(fmt, pages, table, lengths, head_dim, weights, new_table, keep, recent, stream):
    r = _kv_native.kv_evict(_KV_FORMATS.index(fmt), pages, table, lengths, head_dim, weights, new_table, keep, recent, _handle(stream))
    if r.__class__ is not int:
        return r
    if r > 0:
        raise TorqError(r, f"torq_{fmt}_kv_evict")
    cache = _kv_cache(fmt, pages, table, lengths, head_dim, (1.0, 1.0), None, table.shape[0] if isinstance(table, torch.Tensor) else 0)
    _operand(weights, (torch.float32,), "weights", (cache.num_pages, cache.kv_heads, cache.page_tokens))
    _operand(new_table, _INTS, "new_table")
    if new_table.dim() != 2 or new_table.shape[0] != cache.batch:
        raise ValueError(f"new_table: expected a row for each of {cache.batch} sequences, got {tuple(new_table.shape)}")
    name = f"torq_{fmt}_kv_evict"
    if keep < 1:
        raise ValueError(f"{name}: keep has to be positive, got {keep}")
    new_lengths = torch.empty(cache.batch, dtype=torch.int32, device=pages.device)
    kept = torch.empty((cache.batch, cache.kv_heads, keep), dtype=torch.int32, device=pages.device)
    _used_by(stream, new_lengths, kept)
    _raise(getattr(lib(), name)(cache, _ptr(weights), _ptr(new_table), new_table.shape[1], keep, recent, _ptr(new_lengths), _ptr(kept),
                                _stream(stream)), name)
    return new_lengths, kept


def torq_mxfp4_kv_append(pages, table, lengths, K, V, starts=None, stream=None):
    """New keys and values K, V [tokens, kv_heads, dim] float32 or bfloat16 (rows may lie apart) into their slots in pages."""
    _kv_append("mxfp4", pages, table, lengths, K, V, None, starts, stream)


def torq_nvfp4_kv_append(pages, table, lengths, K, V, k_tensor_scale: float, v_tensor_scale: float, starts=None, stream=None):
    """The same in NVFP4."""
    _kv_append("nvfp4", pages, table, lengths, K, V, (k_tensor_scale, v_tensor_scale), starts, stream)


def torq_mxint4_kv_append(pages, table, lengths, K, V, starts=None, stream=None):
    """The same in MXINT4."""
    _kv_append("mxint4", pages, table, lengths, K, V, None, starts, stream)


def torq_mxfp4_kv_read(pages, table, lengths, head_dim: int, tokens: int, starts=None, out_dtype=torch.bfloat16, stream=None):
    """The last `tokens` tokens of the sequences (one of each, or as starts says): (K, V) [tokens, kv_heads, dim]."""
    return _kv_read("mxfp4", pages, table, lengths, head_dim, tokens, None, starts, out_dtype, stream)


def torq_nvfp4_kv_read(pages, table, lengths, head_dim: int, tokens: int, k_tensor_scale: float, v_tensor_scale: float, starts=None,
                       out_dtype=torch.bfloat16, stream=None):
    """The same from NVFP4."""
    return _kv_read("nvfp4", pages, table, lengths, head_dim, tokens, (k_tensor_scale, v_tensor_scale), starts, out_dtype, stream)


def torq_mxint4_kv_read(pages, table, lengths, head_dim: int, tokens: int, starts=None, out_dtype=torch.bfloat16, stream=None):
    """The same from MXINT4."""
    return _kv_read("mxint4", pages, table, lengths, head_dim, tokens, None, starts, out_dtype, stream)


def torq_mxfp4_kv_attention(pages, table, lengths, Q, starts=None, scale=None, softcap: float = 0.0, slopes=None, window: int = 0, prefix=None,
                            first=None, out=None, return_lse: bool = False, workspace=None, stream=None):
    """Attention of Q [tokens, heads, dim] bf16 over the cached tokens of its sequences -> out [tokens, heads, dim] bf16, or (out, lse).
    scale: dim ** -0.5; softcap, slopes, window, prefix, first: torq_kv_scoring."""
    return _kv_attention("mxfp4", pages, table, lengths, Q, None, starts, scale, softcap, slopes, window, prefix, first, out, return_lse,
                         workspace, stream)


def torq_nvfp4_kv_attention(pages, table, lengths, Q, k_tensor_scale: float, v_tensor_scale: float, starts=None, scale=None,
                            softcap: float = 0.0, slopes=None, window: int = 0, prefix=None, first=None, out=None, return_lse: bool = False,
                            workspace=None, stream=None):
    """The same over an NVFP4 cache."""
    return _kv_attention("nvfp4", pages, table, lengths, Q, (k_tensor_scale, v_tensor_scale), starts, scale, softcap, slopes, window, prefix,
                         first, out, return_lse, workspace, stream)


def torq_mxint4_kv_attention(pages, table, lengths, Q, starts=None, scale=None, softcap: float = 0.0, slopes=None, window: int = 0,
                             prefix=None, first=None, out=None, return_lse: bool = False, workspace=None, stream=None):
    """The same over an MXINT4 cache."""
    return _kv_attention("mxint4", pages, table, lengths, Q, None, starts, scale, softcap, slopes, window, prefix, first, out, return_lse,
                         workspace, stream)


def torq_mxfp4_kv_weights(pages, table, lengths, Q, lse, weights, starts=None, scale=None, softcap: float = 0.0, slopes=None,
                          window: int = 0, prefix=None, first=None, weights_out=None, stream=None):
    """What attention (same arguments, its lse) gave to each cached token, added to weights [num_pages, kv_heads, page_tokens] float32
    (a new token's starts at zero): in place, or to weights_out.  No two sequences of a call share a page: those that do get calls of their own."""
    return _kv_weights("mxfp4", pages, table, lengths, Q, lse, weights, None, starts, scale, softcap, slopes, window, prefix, first,
                       weights_out, stream)


def torq_nvfp4_kv_weights(pages, table, lengths, Q, lse, weights, k_tensor_scale: float, starts=None, scale=None, softcap: float = 0.0,
                          slopes=None, window: int = 0, prefix=None, first=None, weights_out=None, stream=None):
    """The same of an NVFP4 cache."""
    return _kv_weights("nvfp4", pages, table, lengths, Q, lse, weights, (k_tensor_scale, 1.0), starts, scale, softcap, slopes, window,
                       prefix, first, weights_out, stream)


def torq_mxint4_kv_weights(pages, table, lengths, Q, lse, weights, starts=None, scale=None, softcap: float = 0.0, slopes=None,
                           window: int = 0, prefix=None, first=None, weights_out=None, stream=None):
    """The same of an MXINT4 cache."""
    return _kv_weights("mxint4", pages, table, lengths, Q, lse, weights, None, starts, scale, softcap, slopes, window, prefix, first,
                       weights_out, stream)


def torq_mxfp4_kv_evict(pages, table, lengths, head_dim: int, weights, new_table, keep: int, recent: int = 0, stream=None):
    """The `recent` newest tokens of each sequence and head and those of the others with the largest weights, `keep` in all, moved to the
    pages of new_table [batch, width], their weights with them -> (new lengths [batch], places that stayed [batch, kv_heads, keep])."""
    return _kv_evict("mxfp4", pages, table, lengths, head_dim, weights, new_table, keep, recent, stream)


def torq_nvfp4_kv_evict(pages, table, lengths, head_dim: int, weights, new_table, keep: int, recent: int = 0, stream=None):
    """The same of an NVFP4 cache."""
    return _kv_evict("nvfp4", pages, table, lengths, head_dim, weights, new_table, keep, recent, stream)


def torq_mxint4_kv_evict(pages, table, lengths, head_dim: int, weights, new_table, keep: int, recent: int = 0, stream=None):
    """The same of an MXINT4 cache."""
    return _kv_evict("mxint4", pages, table, lengths, head_dim, weights, new_table, keep, recent, stream)


# ---- calibration of the inter-block rotation (Section 5.1, Algorithm 1; offline) -----------------------
def torq_block_covariance(X, out=None, stream=None):
    """X [T,d] bf16 -> Sigma [d/32,d/32] float64: covariance across blocks, pooled over tokens and positions."""
    _check(X, torch.bfloat16, "X")
    T, d = X.shape
    if out is None:
        out = torch.empty((d // 32, d // 32), dtype=torch.float64, device=X.device)
    _check(out, torch.float64, "out")
    _raise(lib().torq_block_covariance(_ptr(X), T, d, _ptr(out), _stream(stream)), "torq_block_covariance")
    return out


def torq_givens_equalize(Sigma, eps: float, stream=None):
    """Algorithm 1 on Sigma [B,B] float64 (overwritten with Q Sigma Q^T).
    Returns (Q float64 [B,B], Q bf16 [B,B], number of rotations as a device int32 tensor)."""
    _check(Sigma, torch.float64, "Sigma")
    B = Sigma.shape[0]
    Q = torch.empty((B, B), dtype=torch.float64, device=Sigma.device)
    Qb = torch.empty((B, B), dtype=torch.bfloat16, device=Sigma.device)
    n = torch.zeros(4, dtype=torch.int32, device=Sigma.device)
    _raise(lib().torq_givens_equalize(_ptr(Sigma), B, float(eps), _ptr(Q), _ptr(Qb), _ptr(n), _stream(stream)),
           "torq_givens_equalize")
    return Q, Qb, n[:1]


def torq_rotate_quantize_structured_nvfp4(X, R_B, R_intra, tensor_scale: float, out_codes=None, out_scales=None,
                                          stream=None):
    """The structured rotation (R_B [d/32,d/32], shared R_intra [32,32] or None) followed by the NVFP4 quantizer."""
    M, d = X.shape
    for t, n in ((X, "X"), (R_B, "R_B"), (R_intra, "R_intra")):
        _check(t, torch.bfloat16, n)
    if out_codes is None:
        out_codes = torch.empty((M, d // 2), dtype=torch.uint8, device=X.device)
    if out_scales is None:
        out_scales = torch.empty(torq_nvfp4_scales_bytes(M, d), dtype=torch.uint8, device=X.device)
    _raise(lib().torq_rotate_quantize_structured_nvfp4(_ptr(X), _ptr(R_B), _ptr(R_intra), M, d, tensor_scale,
                                                       _ptr(out_codes), _ptr(out_scales), _stream(stream)),
           "torq_rotate_quantize_structured_nvfp4")
    return out_codes, out_scales
