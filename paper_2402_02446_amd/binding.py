"""ctypes face of liblqer.so: same names as the C ABI in include/lqer.h.

Argument marshalling only: every step of the layer runs in the library's HIP
kernels.  PyTorch supplies device memory and the current HIP stream.  There is
no fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblqer.so")

LQER_OK = 0
STATUS_NAMES = {0: "LQER_OK", 1: "LQER_ERR_NULL", 2: "LQER_ERR_SHAPE", 3: "LQER_ERR_UNSUPPORTED",
                4: "LQER_ERR_SINGULAR_SCALE", 5: "LQER_ERR_WORKSPACE", 6: "LQER_ERR_HIP",
                7: "LQER_ERR_NO_CONVERGENCE", 8: "LQER_ERR_VALUE", 9: "LQER_ERR_NO_MEMORY"}

# every symbol include/lqer.h declares
EXPORTS = ("lqer_status_string", "lqer_quantize_mx", "lqer_build_factors", "lqer_build_factors_device",
           "lqer_layer_import",
           "lqer_layer_export", "lqer_layer_dims", "lqer_layer_set_activation_bits", "lqer_layer_fp6_bytes", "lqer_layer_drop_fp6", "lqer_layer_free", "lqer_linear_workspace_bytes", "lqer_linear_workspace_bytes_ex",
           "lqer_linear_forward", "lqer_linear_forward_q", "lqer_linear_forward_ex", "lqer_linear_forward_requant", "lqer_linear_path",
           "lqer_linear_shared_workspace_bytes", "lqer_linear_forward_shared", "lqer_set_wait_limit",
           "lqer_linear_forward_static", "lqer_layer_import_w", "lqer_layer_weight_bits",
           "lqer_int_layer_import", "lqer_int_layer_export", "lqer_quantize_int8_token", "lqer_selftest_layouts",
           "lqer_rmsnorm_mx", "lqer_adapters_workspace_bytes", "lqer_adapters_forward",
           "lqer_kv4_page_bytes", "lqer_kv4_append", "lqer_kv4_attention_workspace_bytes", "lqer_kv4_attention")


class LqerError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


class LaunchOpts(C.Structure):
    _fields_ = [("path", C.c_int), ("variant", C.c_int), ("stages", C.c_int)]


class Kv4Shape(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_requests", "q_heads", "kv_heads", "head_dim", "page_tokens", "table_ld")] + \
               [(n, C.c_int64) for n in ("pages", "Tq", "ldq", "ldo")] + \
               [(n, C.c_int) for n in ("max_q", "max_kv", "causal", "window")] + [("scale", C.c_float), ("out_type", C.c_int)]


class Config(C.Structure):
    _fields_ = [("w_bits", C.c_int), ("h_bits", C.c_int), ("exp_bits", C.c_int), ("block", C.c_int)]


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    # PyTorch ships its own HIP runtime: import it first so that liblqer.so binds to the same
    # runtime instance (and the same streams and allocations) instead of loading a second one.
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2402_02446_amd.build` "
                           "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
    L.lqer_status_string.restype = C.c_char_p
    L.lqer_status_string.argtypes = [i32]
    L.lqer_quantize_mx.restype = i32
    L.lqer_quantize_mx.argtypes = [vp, i64, i64, i64, i32, i32, vp, vp, vp]
    L.lqer_build_factors.restype = i32
    L.lqer_build_factors.argtypes = [vp, i64, i64, vp, i64, i64, i32, i32, vp, C.POINTER(vp)]
    L.lqer_build_factors_device.restype = i32
    L.lqer_build_factors_device.argtypes = [vp, i64, i64, vp, i64, i64, i32, i32, vp, vp, C.POINTER(vp)]
    L.lqer_layer_import.restype = i32
    L.lqer_layer_import.argtypes = [i64, i64, i32, vp, vp, vp, vp, vp, vp, C.POINTER(vp)]
    L.lqer_layer_import_w.restype = i32
    L.lqer_layer_import_w.argtypes = [i32, i64, i64, i32, vp, vp, vp, vp, vp, vp, C.POINTER(vp)]
    L.lqer_layer_weight_bits.restype = i32
    L.lqer_layer_weight_bits.argtypes = [vp]
    L.lqer_int_layer_import.restype = i32
    L.lqer_int_layer_import.argtypes = [i64, i64, i32, vp, vp, vp, vp, vp, vp, C.POINTER(vp)]
    L.lqer_int_layer_export.restype = i32
    L.lqer_int_layer_export.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.lqer_quantize_int8_token.restype = i32
    L.lqer_quantize_int8_token.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    L.lqer_layer_export.restype = i32
    L.lqer_layer_export.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.lqer_layer_dims.restype = i32
    L.lqer_layer_dims.argtypes = [vp, C.POINTER(i64), C.POINTER(i64), C.POINTER(i32), C.POINTER(i32)]
    L.lqer_layer_set_activation_bits.restype = i32
    L.lqer_layer_set_activation_bits.argtypes = [vp, i32]
    L.lqer_layer_fp6_bytes.restype = sz
    L.lqer_layer_fp6_bytes.argtypes = [vp]
    L.lqer_layer_drop_fp6.restype = i32
    L.lqer_layer_drop_fp6.argtypes = [vp]
    L.lqer_layer_free.restype = i32
    L.lqer_layer_free.argtypes = [vp]
    L.lqer_linear_workspace_bytes.restype = sz
    L.lqer_linear_workspace_bytes.argtypes = [vp, i64]
    L.lqer_linear_workspace_bytes_ex.restype = sz
    L.lqer_linear_workspace_bytes_ex.argtypes = [vp, i64, i32]
    L.lqer_linear_forward.restype = i32
    L.lqer_linear_forward.argtypes = [vp, vp, i64, i64, vp, i64, vp, sz, vp]
    L.lqer_linear_forward_q.restype = i32
    L.lqer_linear_forward_q.argtypes = [vp, vp, vp, i64, vp, i64, vp, sz, vp]
    L.lqer_linear_forward_ex.restype = i32
    L.lqer_linear_forward_ex.argtypes = [vp, vp, i64, i64, vp, i64, vp, sz, vp, C.POINTER(LaunchOpts)]
    L.lqer_linear_forward_requant.restype = i32
    L.lqer_linear_forward_requant.argtypes = [vp, vp, i64, i64, vp, i64, vp, vp, sz, vp, vp]
    L.lqer_linear_shared_workspace_bytes.restype = sz
    L.lqer_linear_shared_workspace_bytes.argtypes = [C.POINTER(vp), i32, i64]
    L.lqer_linear_forward_shared.restype = i32
    L.lqer_linear_forward_shared.argtypes = [C.POINTER(vp), i32, vp, i64, i64, C.POINTER(vp), C.POINTER(i64), vp, sz, vp]
    L.lqer_set_wait_limit.restype = i32
    L.lqer_set_wait_limit.argtypes = [i32]
    L.lqer_linear_path.restype = i32
    L.lqer_linear_path.argtypes = [vp, i64]
    L.lqer_linear_forward_static.restype = i32
    L.lqer_linear_forward_static.argtypes = [vp, vp, i64, i64, vp, i64, vp]
    f32 = C.c_float
    L.lqer_rmsnorm_mx.restype = i32
    L.lqer_rmsnorm_mx.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, i32, vp, i32, f32, i32, vp, vp, vp, i64, vp]
    L.lqer_adapters_workspace_bytes.restype = sz
    L.lqer_adapters_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    L.lqer_adapters_forward.restype = i32
    L.lqer_adapters_forward.argtypes = [vp, i64, i64, i64, vp, vp, vp, i32, i32, vp, vp, vp, i64, vp, i64, i64, vp, sz, vp]
    L.lqer_kv4_page_bytes.restype = sz
    L.lqer_kv4_page_bytes.argtypes = [i32, i32]
    L.lqer_kv4_append.restype = i32
    L.lqer_kv4_append.argtypes = [vp, i64, i32, i32, i32, vp, i64, vp, i64, i32, i64, vp, vp]
    L.lqer_kv4_attention_workspace_bytes.restype = sz
    L.lqer_kv4_attention_workspace_bytes.argtypes = [C.POINTER(Kv4Shape)]
    L.lqer_kv4_attention.restype = i32
    L.lqer_kv4_attention.argtypes = [C.POINTER(Kv4Shape), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    _lib = L
    return L


def _check(status: int, where: str):
    if status != LQER_OK:
        raise LqerError(status, where)


def _np_ptr(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _stream():
    """The handle of torch's current stream on the current device.  Asked for by number: the Stream object that
    torch.cuda.current_stream() builds around it takes 2.7 us, a quarter of a few-token call; this takes 0.2."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def lqer_status_string(status: int) -> str:
    return lib().lqer_status_string(int(status)).decode()


def lqer_quantize_mx(x, elem_bits: int = 8, exp_bits: int = 8):
    """x: CUDA fp32 [rows][cols] (row stride may exceed cols). Returns (codes, exps) CUDA tensors."""
    import torch
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    code_cols = cols if elem_bits >= 6 else cols // 2
    codes = torch.empty((rows, code_cols), dtype=torch.int8 if elem_bits >= 6 else torch.uint8, device=x.device)
    exps = torch.empty((rows, cols // 16), dtype=torch.uint8, device=x.device)
    _check(lib().lqer_quantize_mx(x.data_ptr(), rows, cols, ld, elem_bits, exp_bits,
                                  codes.data_ptr(), exps.data_ptr(), _stream()),
           "lqer_quantize_mx")
    return codes, exps


class Layer:
    """Owning wrapper of an lqer_layer handle."""

    def __init__(self, handle):
        self.handle = C.c_void_p(handle)
        K, N, k, kp = C.c_int64(), C.c_int64(), C.c_int(), C.c_int()
        _check(lib().lqer_layer_dims(self.handle, C.byref(K), C.byref(N), C.byref(k), C.byref(kp)),
               "lqer_layer_dims")
        self.K, self.N, self.k, self.kp = K.value, N.value, k.value, kp.value
        self.w_bits = int(lib().lqer_layer_weight_bits(self.handle))
        self._ws = None

    def set_activation_bits(self, bits: int):
        _check(lib().lqer_layer_set_activation_bits(self.handle, int(bits)), "lqer_layer_set_activation_bits")

    def fp6_bytes(self) -> int:
        return int(lib().lqer_layer_fp6_bytes(self.handle))

    def drop_fp6(self):
        _check(lib().lqer_layer_drop_fp6(self.handle), "lqer_layer_drop_fp6")

    def free(self):
        if self.handle:
            lib().lqer_layer_free(self.handle)
            self.handle = C.c_void_p(None)
            self._ws = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def workspace(self, M: int, path: int = 0):
        """A cached torch allocation of lqer_linear_workspace_bytes_ex(M, path) bytes."""
        import torch
        need = lib().lqer_linear_workspace_bytes_ex(self.handle, M, path)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        return self._ws


def lqer_layer_import(K, N, k, Wc, We, Ac=None, Ae=None, Bc=None, Be=None) -> Layer:
    arrs = [None if a is None else np.ascontiguousarray(a) for a in (Wc, We, Ac, Ae, Bc, Be)]
    out = C.c_void_p()
    _check(lib().lqer_layer_import(K, N, k, *[_np_ptr(a) for a in arrs], C.byref(out)), "lqer_layer_import")
    return Layer(out.value)


def lqer_layer_import_w(w_bits, K, N, k, Wc, We, Ac=None, Ae=None, Bc=None, Be=None) -> Layer:
    """Import with the mantissa width of W_q given: 4 (Wc [N][K/2]) or 2 (Wc [N][K/4])."""
    arrs = [None if a is None else np.ascontiguousarray(a) for a in (Wc, We, Ac, Ae, Bc, Be)]
    if arrs[0].size != N * K * w_bits // 8:
        raise ValueError("Wc does not hold N * K codes of that width")
    out = C.c_void_p()
    _check(lib().lqer_layer_import_w(int(w_bits), K, N, k, *[_np_ptr(a) for a in arrs], C.byref(out)), "lqer_layer_import_w")
    return Layer(out.value)


def lqer_int_layer_import(K, N, k, Wc, Ws, Ac=None, As=None, Bc=None, Bs=None) -> Layer:
    """INT layer from canonical arrays; scales are float16 arrays."""
    arrs = [np.ascontiguousarray(Wc, dtype=np.uint8), np.ascontiguousarray(Ws, dtype=np.float16)]
    for a, dt in ((Ac, np.int8), (As, np.float16), (Bc, np.int8), (Bs, np.float16)):
        arrs.append(None if (a is None or k == 0) else np.ascontiguousarray(a, dtype=dt))
    out = C.c_void_p()
    _check(lib().lqer_int_layer_import(K, N, k, *[_np_ptr(a) for a in arrs], C.byref(out)), "lqer_int_layer_import")
    return Layer(out.value)


def lqer_int_layer_export(layer: Layer):
    K, N, kp = layer.K, layer.N, layer.kp
    Wc, Ws = np.zeros((N, K // 2), np.uint8), np.zeros((N, K // 128), np.float16)
    Ac, As = np.zeros((kp, K), np.int8), np.zeros((kp, K // 128), np.float16)
    Bc, Bs = np.zeros((N, kp), np.int8), np.zeros((N,), np.float16)
    ptrs = [_np_ptr(a) for a in ((Wc, Ws, Ac, As, Bc, Bs) if kp else (Wc, Ws))] + ([] if kp else [None] * 4)
    _check(lib().lqer_int_layer_export(layer.handle, *ptrs), "lqer_int_layer_export")
    return dict(Wc=Wc, Ws=Ws, Ac=Ac, As=As, Bc=Bc, Bs=Bs)


def lqer_quantize_int8_token(x):
    """x: CUDA fp32 [rows][cols].  Returns (codes int8 [rows][cols], scales float16 [rows]) CUDA tensors."""
    import torch
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    codes = torch.empty((rows, cols), dtype=torch.int8, device=x.device)
    scales = torch.empty((rows,), dtype=torch.float16, device=x.device)
    _check(lib().lqer_quantize_int8_token(x.data_ptr(), rows, cols, ld, codes.data_ptr(),
                                          scales.data_ptr(), _stream()), "lqer_quantize_int8_token")
    return codes, scales


def lqer_layer_export(layer: Layer):
    K, N, kp = layer.K, layer.N, layer.kp
    Wc = np.zeros((N, K * layer.w_bits // 8), np.uint8)
    We = np.zeros((N, K // 16), np.uint8)
    Ac = np.zeros((kp, K), np.int8)
    Ae = np.zeros((kp, K // 16), np.uint8)
    Bc = np.zeros((N, kp), np.int8)
    Be = np.zeros((N, kp // 16), np.uint8)
    _check(lib().lqer_layer_export(layer.handle, *[_np_ptr(a) for a in (Wc, We, Ac, Ae, Bc, Be)]),
           "lqer_layer_export")
    return dict(Wc=Wc, We=We, Ac=Ac, Ae=Ae, Bc=Bc, Be=Be)


def lqer_build_factors(W, calib, k: int, mode: int = 1, cfg=None) -> Layer:
    W = np.ascontiguousarray(W, dtype=np.float32)
    K, N = W.shape
    if calib is not None:
        calib = np.ascontiguousarray(calib, dtype=np.float32)
        ns, rows, kc = calib.shape
        if kc != K:
            raise ValueError("calib's last axis must be K")
    else:
        ns, rows = 0, 0
    c = None if cfg is None else C.byref(Config(*cfg))
    out = C.c_void_p()
    _check(lib().lqer_build_factors(_np_ptr(W), K, N, _np_ptr(calib), ns, rows, k, mode, c, C.byref(out)),
           "lqer_build_factors")
    return Layer(out.value)


def lqer_build_factors_device(W, calib, k: int, mode: int = 1, cfg=None) -> Layer:
    """W [K][N] and calib [n_samples][rows][K] are fp32 CUDA tensors; runs on torch's current stream."""
    import torch
    if not (W.is_cuda and W.dtype == torch.float32 and (calib is None or (calib.is_cuda and calib.dtype == torch.float32))):
        raise ValueError("W and calib must be fp32 CUDA tensors")
    W = W.contiguous()
    K, N = W.shape
    if calib is not None:
        calib = calib.contiguous()
        ns, rows, kc = calib.shape
        if kc != K:
            raise ValueError("calib's last axis must be K")
        cptr = calib.data_ptr()
    else:
        ns, rows, cptr = 0, 0, None
    c = None if cfg is None else C.byref(Config(*cfg))
    out = C.c_void_p()
    _check(lib().lqer_build_factors_device(W.data_ptr(), K, N, cptr, ns, rows, k, mode, c, _stream(), C.byref(out)),
           "lqer_build_factors_device")
    return Layer(out.value)


def lqer_linear_workspace_bytes(layer: Layer, M: int, path: int = 0) -> int:
    return int(lib().lqer_linear_workspace_bytes_ex(layer.handle, M, path))


def lqer_linear_path(layer: Layer, M: int) -> int:
    return int(lib().lqer_linear_path(layer.handle, M))


def lqer_linear_forward(layer: Layer, X, Y=None, workspace=None):
    M = X.shape[0]
    if Y is None:
        import torch
        Y = torch.empty((M, layer.N), dtype=torch.float32, device=X.device)
    ws = layer.workspace(M) if workspace is None else workspace
    ldx = X.stride(0) if M > 1 else max(layer.K, X.stride(0))
    ldy = Y.stride(0) if M > 1 else max(layer.N, Y.stride(0))
    _check(lib().lqer_linear_forward(layer.handle, X.data_ptr(), M, ldx, Y.data_ptr(),
                                     ldy, ws.data_ptr(), ws.numel(), _stream()),
           "lqer_linear_forward")
    return Y


def lqer_linear_forward_static(layer: Layer, X, Y=None):
    """The forward pass on the library's own static scratch (no workspace argument)."""
    M = X.shape[0]
    if Y is None:
        import torch
        Y = torch.empty((M, layer.N), dtype=torch.float32, device=X.device)
    ldx = X.stride(0) if M > 1 else max(layer.K, X.stride(0))
    ldy = Y.stride(0) if M > 1 else max(layer.N, Y.stride(0))
    _check(lib().lqer_linear_forward_static(layer.handle, X.data_ptr(), M, ldx, Y.data_ptr(),
                                            ldy, _stream()),
           "lqer_linear_forward_static")
    return Y


def lqer_linear_forward_q(layer: Layer, Xc, Xe, Y=None, workspace=None):
    M = Xc.shape[0]
    if Y is None:
        import torch
        Y = torch.empty((M, layer.N), dtype=torch.float32, device=Xc.device)
    ws = layer.workspace(M) if workspace is None else workspace
    ldy = Y.stride(0) if M > 1 else max(layer.N, Y.stride(0))
    _check(lib().lqer_linear_forward_q(layer.handle, Xc.data_ptr(), Xe.data_ptr(), M,
                                       Y.data_ptr(), ldy, ws.data_ptr(), ws.numel(),
                                       _stream()),
           "lqer_linear_forward_q")
    return Y


def lqer_linear_forward_ex(layer: Layer, X, Y=None, workspace=None, path=0, variant=0, stages=0):
    M = X.shape[0]
    if Y is None:
        import torch
        Y = torch.empty((M, layer.N), dtype=torch.float32, device=X.device)
    ws = layer.workspace(M, path) if workspace is None else workspace
    ldx = X.stride(0) if M > 1 else max(layer.K, X.stride(0))
    ldy = Y.stride(0) if M > 1 else max(layer.N, Y.stride(0))
    opts = LaunchOpts(path, variant, stages)
    _check(lib().lqer_linear_forward_ex(layer.handle, X.data_ptr(), M, ldx,
                                        Y.data_ptr(), ldy, ws.data_ptr(), ws.numel(),
                                        _stream(), C.byref(opts)),
           "lqer_linear_forward_ex")
    return Y


def lqer_linear_forward_requant(layer: Layer, X, workspace=None, path=0, variant=0):
    """Forward pass with Y leaving as MXINT8: returns (codes int8 [M][N], exps uint8 [M][N/16])."""
    import torch
    M = X.shape[0]
    codes = torch.empty((M, layer.N), dtype=torch.int8, device=X.device)
    exps = torch.empty((M, layer.N // 16), dtype=torch.uint8, device=X.device)
    ws = layer.workspace(M, path) if workspace is None else workspace
    ldx = X.stride(0) if M > 1 else max(layer.K, X.stride(0))
    opts = LaunchOpts(path, variant, 0)
    _check(lib().lqer_linear_forward_requant(layer.handle, X.data_ptr(), M, ldx,
                                             codes.data_ptr(), layer.N, exps.data_ptr(),
                                             ws.data_ptr(), ws.numel(), _stream(), C.byref(opts)),
           "lqer_linear_forward_requant")
    return codes, exps


def lqer_linear_shared_workspace_bytes(layers, M: int) -> int:
    arr = (C.c_void_p * len(layers))(*[l.handle for l in layers])
    return int(lib().lqer_linear_shared_workspace_bytes(arr, len(layers), M))


def lqer_linear_forward_shared(layers, X, Ys=None, workspace=None):
    """Several layers applied to the same X (quantized once): returns the list of their Y."""
    import torch
    M = X.shape[0]
    n = len(layers)
    if Ys is None:
        Ys = [torch.empty((M, l.N), dtype=torch.float32, device=X.device) for l in layers]
    arr = (C.c_void_p * n)(*[l.handle for l in layers])
    if workspace is None:
        need = lib().lqer_linear_shared_workspace_bytes(arr, n, M)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    ldx = X.stride(0) if M > 1 else max(layers[0].K, X.stride(0))
    yarr = (C.c_void_p * n)(*[y.data_ptr() for y in Ys])
    ldys = (C.c_int64 * n)(*[(y.stride(0) if M > 1 else max(l.N, y.stride(0))) for y, l in zip(Ys, layers)])
    _check(lib().lqer_linear_forward_shared(arr, n, X.data_ptr(), M, ldx, yarr, ldys,
                                            workspace.data_ptr(), workspace.numel(), _stream()),
           "lqer_linear_forward_shared")
    return Ys


def lqer_set_wait_limit(polls: int):
    _check(lib().lqer_set_wait_limit(int(polls)), "lqer_set_wait_limit")


# ---- between a block's linears ------------------------------------------------------------------------------------------
# The C ABI sees pointers only: what a tensor holds, how it is laid out, and that it is on the GPU, is checked here.  These
# calls take a few microseconds on the GPU for single tokens, so the checks are written to cost little: one condition a tensor.
def _refuse(name, what):
    raise ValueError(f"{name} must be {what}")


def _stride(t, rows, cols):
    """The row stride of a matrix; a single row has none of its own, and goes by one that the library takes."""
    return t.stride(0) if rows > 1 else (cols + 7) & -8


def lqer_rmsnorm_mx(x, weight, eps: float = 1e-5, residual=None, h_out=None, elem_bits: int = 8, values: bool = False):
    """x [rows][cols], residual (or None) of x's shape, weight [cols]: fp32 or bf16 CUDA tensors.  Returns (codes int8, exps uint8,
    h, values): h is h_out (a new tensor of residual's type unless given; residual itself updates in place), None without a residual;
    values is the bf16 tensor of what the codes stand for, or None."""
    import torch
    L, f32, bf16 = _lib or lib(), torch.float32, torch.bfloat16
    shape = x.shape
    if len(shape) != 2 or not x.is_cuda or x.dtype not in (f32, bf16) or (x.stride(1) != 1 and shape[1] > 1):
        _refuse("x", "fp32 or bf16 [rows][cols] on the GPU, its rows contiguous")
    rows, cols = shape
    if weight.shape != (cols,) or not weight.is_cuda or weight.dtype not in (f32, bf16) or not weight.is_contiguous():
        _refuse("weight", f"a contiguous fp32 or bf16 [{cols}] on the GPU")
    h = None
    r_ptr = h_ptr = None
    ldr = ldh = res_type = 0
    if residual is not None:
        if residual.shape != shape or not residual.is_cuda or residual.dtype not in (f32, bf16) or (residual.stride(1) != 1 and cols > 1):
            _refuse("residual", "fp32 or bf16 of x's shape on the GPU, its rows contiguous")
        h = residual.new_empty(shape) if h_out is None else h_out
        if h.shape != shape or not h.is_cuda or h.dtype != residual.dtype or (h.stride(1) != 1 and cols > 1):
            _refuse("h_out", "of residual's shape and type, on the GPU, its rows contiguous")
        r_ptr, h_ptr, ldr, ldh, res_type = residual.data_ptr(), h.data_ptr(), _stride(residual, rows, cols), _stride(h, rows, cols), h.dtype == bf16
    codes = torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format)
    exps = x.new_empty((rows, cols // 16), dtype=torch.uint8)
    v = torch.empty_like(codes, dtype=bf16) if values else None
    st = L.lqer_rmsnorm_mx(x.data_ptr(), x.dtype == bf16, rows, cols, _stride(x, rows, cols), r_ptr, ldr, h_ptr, ldh, res_type,
                           weight.data_ptr(), weight.dtype == bf16, eps, elem_bits, codes.data_ptr(), exps.data_ptr(),
                           v.data_ptr() if values else None, cols, _stream())
    if st:
        raise LqerError(st, "lqer_rmsnorm_mx")
    return codes, exps, h, v


@functools.lru_cache(maxsize=256)
def lqer_adapters_workspace_bytes(M: int, K: int, N: int, R: int, n_adapters: int) -> int:
    return int(lib().lqer_adapters_workspace_bytes(M, K, N, R, n_adapters))


def lqer_adapters_forward(X, ids, A, B, Y, out=None, ranks=None, scales=None, workspace=None):
    """Y + the adapters of every token: X bf16 [M][K], ids int32 [M], A bf16 [n][R][K], B bf16 [n][N][R], Y fp32 [M][N]; ranks int32 [n],
    scales fp32 [n].  The result is written to `out` (Y itself unless given) and returned."""
    import torch
    L, bf16, f32, i32 = _lib or lib(), torch.bfloat16, torch.float32, torch.int32
    n, R, K = A.shape
    M, N = shape = Y.shape
    if A.dtype is not bf16 or not A.is_cuda or not A.is_contiguous():
        _refuse("A", "a contiguous bf16 [adapters][rank][K] on the GPU")
    if B.shape != (n, N, R) or B.dtype is not bf16 or not B.is_cuda or not B.is_contiguous():
        _refuse("B", f"a contiguous bf16 [{n}][{N}][{R}] on the GPU")
    if X.shape != (M, K) or X.dtype is not bf16 or not X.is_cuda or (X.stride(1) != 1 and K > 1):
        _refuse("X", f"bf16 [{M}][{K}] on the GPU, its rows contiguous")
    if Y.dtype is not f32 or not Y.is_cuda or (Y.stride(1) != 1 and N > 1):
        _refuse("Y", "fp32 [tokens][N] on the GPU, its rows contiguous")
    if out is None:
        out = Y
    elif out.shape != shape or out.dtype is not f32 or not out.is_cuda or (out.stride(1) != 1 and N > 1):
        _refuse("out", "fp32 of Y's shape on the GPU, its rows contiguous")
    if ids.shape != (M,) or ids.dtype is not i32 or not ids.is_cuda or not ids.is_contiguous():
        _refuse("ids", f"a contiguous int32 [{M}] on the GPU")
    if ranks is not None and (ranks.shape != (n,) or ranks.dtype is not i32 or not ranks.is_cuda or not ranks.is_contiguous()):
        _refuse("ranks", f"a contiguous int32 [{n}] on the GPU")
    if scales is not None and (scales.shape != (n,) or scales.dtype is not f32 or not scales.is_cuda or not scales.is_contiguous()):
        _refuse("scales", f"a contiguous fp32 [{n}] on the GPU")
    if workspace is None:
        workspace = X.new_empty(max(lqer_adapters_workspace_bytes(M, K, N, R, n), 256), dtype=torch.uint8)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        _refuse("workspace", "contiguous, on the GPU")
    st = L.lqer_adapters_forward(X.data_ptr(), M, K, _stride(X, M, K), ids.data_ptr(), A.data_ptr(), B.data_ptr(), n, R,
                                 None if ranks is None else ranks.data_ptr(), None if scales is None else scales.data_ptr(),
                                 Y.data_ptr(), _stride(Y, M, N), out.data_ptr(), N, _stride(out, M, N),
                                 workspace.data_ptr(), workspace.nbytes, _stream())
    if st:
        raise LqerError(st, "lqer_adapters_forward")
    return out


def lqer_kv4_page_bytes(page_tokens: int, head_dim: int) -> int:
    return int(lib().lqer_kv4_page_bytes(page_tokens, head_dim))


def lqer_kv4_pool(pages: int, kv_heads: int, page_tokens: int, head_dim: int, device="cuda"):
    """An uncleared pool: uint8 [pages][kv_heads][lqer_kv4_page_bytes]."""
    import torch
    size = lqer_kv4_page_bytes(page_tokens, head_dim)
    if size == 0:
        raise LqerError(3, "lqer_kv4_pool")
    return torch.empty((pages, kv_heads, size), dtype=torch.uint8, device=device)


def _kv4_pool(pool, head_dim, u8):
    """(pages, kv_heads, page_tokens) of a pool for heads of that dimension."""
    if pool.dim() != 3 or pool.dtype is not u8 or not pool.is_cuda or not pool.is_contiguous():
        _refuse("pool", "a contiguous uint8 [pages][kv_heads][bytes of a page] on the GPU")
    pages, heads, size = pool.shape
    page_tokens, left = divmod(size * 8, head_dim * 9) if head_dim > 0 else (0, 1)
    if left:
        _refuse("pool", f"of whole tokens of {head_dim} dimensions")
    return pages, heads, page_tokens


def _token_stride(stride, tokens, heads, head_dim):
    """The token stride of [tokens][heads][head_dim] whose heads lie side by side; 0 where they do not."""
    t, h, d = stride
    if d != 1 or (h != head_dim and heads != 1):
        return 0
    return t if tokens > 1 else heads * head_dim


def lqer_kv4_append(pool, k, v, slots):
    """k, v [T][kv_heads][head_dim], both fp32 or both bf16, into the pool's slots (int32 [T]: page * page_tokens + place)."""
    import torch
    L, bf16 = _lib or lib(), torch.bfloat16
    T, heads, D = shape = k.shape
    dtype = k.dtype
    pages, pool_heads, P = _kv4_pool(pool, D, torch.uint8)
    if heads != pool_heads or not k.is_cuda or (dtype is not bf16 and dtype is not torch.float32):
        _refuse("k", f"fp32 or bf16 [tokens][{pool_heads}][head_dim] on the GPU")
    if v.shape != shape or not v.is_cuda or v.dtype is not dtype:
        _refuse("v", "of k's shape and type, on the GPU")
    if slots.shape != (T,) or slots.dtype is not torch.int32 or not slots.is_cuda or not slots.is_contiguous():
        _refuse("slots", f"a contiguous int32 [{T}] on the GPU")
    ldk, ldv = _token_stride(k.stride(), T, heads, D), _token_stride(v.stride(), T, heads, D)
    if not ldk or not ldv:
        _refuse("k and v", "of heads that lie side by side in a token")
    st = L.lqer_kv4_append(pool.data_ptr(), pages, P, heads, D, k.data_ptr(), ldk, v.data_ptr(), ldv, dtype is bf16, T, slots.data_ptr(), _stream())
    if st:
        raise LqerError(st, "lqer_kv4_append")


@functools.lru_cache(maxsize=256)
def _kv4_sizes(*sizes):
    """A call's sizes as the library takes them, the bytes of its workspace, and the requests."""
    shape = Kv4Shape(*sizes)
    max_q, max_kv, _, window = sizes[10:14]
    if not (0 <= max_q < 1 << 31 and 0 <= max_kv < 1 << 31 and 0 <= window < 1 << 31):
        # (ctypes keeps the low 32 bits: a wide window would be a narrow one)
        shape.max_q, shape.max_kv, shape.window = (min(max(n, -1), (1 << 31) - 1) for n in (max_q, max_kv, window))
    return C.byref(shape), int(lib().lqer_kv4_attention_workspace_bytes(C.byref(shape))), shape.n_requests


def _kv4_shape(torch, pool, q, table, max_q, max_kv, scale, causal, window, out):
    Tq, q_heads, D = shape = q.shape
    bf16 = torch.bfloat16
    pages, heads, P = _kv4_pool(pool, D, torch.uint8)
    ldq = _token_stride(q.stride(), Tq, q_heads, D)
    if not ldq or q.dtype is not bf16 or not q.is_cuda:
        _refuse("q", "bf16 [tokens][q_heads][head_dim] on the GPU, a token's heads side by side")
    ldo, out_type = q_heads * D, 1
    if out is not None:
        ldo, out_type = _token_stride(out.stride(), Tq, q_heads, D) if out.shape == shape else 0, out.dtype is bf16
        if not ldo or not out.is_cuda or (not out_type and out.dtype is not torch.float32):
            _refuse("out", "bf16 or fp32 of q's shape on the GPU, a token's heads side by side")
    if table.dim() != 2 or table.dtype is not torch.int32 or not table.is_cuda or not table.is_contiguous():
        _refuse("table", "a contiguous int32 [requests][pages] on the GPU")
    n, ld = table.shape
    return _kv4_sizes(n, q_heads, heads, D, P, ld, pages, Tq, ldq, ldo, max_q, max_kv, bool(causal), window, scale, out_type)


def lqer_kv4_attention_workspace_bytes(pool, q, table, max_q: int, max_kv: int, causal: bool = True, window: int = 0) -> int:
    """Bytes of the workspace of lqer_kv4_attention with tensors and numbers like these."""
    import torch
    return _kv4_shape(torch, pool, q, table, max_q, max_kv, 1.0, causal, window, None)[1]


def lqer_kv4_attention(pool, q, cu_q, kv_len, table, max_q: int, max_kv: int, scale: float, causal: bool = True, window: int = 0, out=None,
                       workspace=None):
    """Attention of q bf16 [Tq][q_heads][head_dim] over the pool: request b has rows cu_q[b] .. cu_q[b + 1] - 1 of q, kv_len[b] cached tokens
    and the pages table[b] (int32 tensors).  Returns out (bf16 unless given, bf16 or fp32)."""
    import torch
    L, i32 = _lib or lib(), torch.int32
    sizes, need, n = _kv4_shape(torch, pool, q, table, max_q, max_kv, scale, causal, window, out)
    if cu_q.shape != (n + 1,) or cu_q.dtype is not i32 or not cu_q.is_cuda or not cu_q.is_contiguous():
        _refuse("cu_q", f"a contiguous int32 [{n + 1}] on the GPU")
    if kv_len.shape != (n,) or kv_len.dtype is not i32 or not kv_len.is_cuda or not kv_len.is_contiguous():
        _refuse("kv_len", f"a contiguous int32 [{n}] on the GPU")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if workspace is None:
        if need:
            workspace = q.new_empty(need, dtype=torch.uint8)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        _refuse("workspace", "contiguous, on the GPU")
    st = L.lqer_kv4_attention(sizes, pool.data_ptr(), q.data_ptr(), cu_q.data_ptr(), kv_len.data_ptr(), table.data_ptr(), out.data_ptr(),
                              None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes, _stream())
    if st:
        raise LqerError(st, "lqer_kv4_attention")
    return out
