"""Python binding of the MI355X SOAP optimizer-step library (libsoap_mi355x.so).

Argument marshalling only: every function forwards to the C entry point of the
same name in ``include/soap.h``; all arithmetic runs in the HIP kernels.
Matrix arguments may be torch tensors (fp32, contiguous, on the GPU) or raw
integer device pointers; ``None`` passes NULL.  The stream defaults to torch's
current stream.  A nonzero status raises ``SoapError`` carrying
``soap_last_error()``.  There is no fallback: if the library is not built,
``lib()`` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsoap_mi355x.so")

SOAP_OK = 0
SOAP_ERR_NULL = -1
SOAP_ERR_SHAPE = -2
SOAP_ERR_HPARAM = -3
SOAP_ERR_WORKSPACE = -4
SOAP_ERR_ALIGN = -5
SOAP_ERR_ALIAS = -6
SOAP_ERR_HIP = -7
SOAP_ERR_QR_GAVE_UP = -8
SOAP_STATUS_QR_L = 1
SOAP_STATUS_QR_R = 2
SOAP_FLAG_NO_BIAS_CORRECTION = 1
SOAP_FLAG_SKIP_REFRESH = 2
SOAP_FLAG_STALE_REFRESH = 4
SOAP_MUON_BF16 = 1
SOAP_MAX_DIM = 16384
SOAP_F32 = 0
SOAP_BF16 = 1
SOAP_MAX_ROWS = 1 << 24
SOAP_ROUTER_RENORMALIZE = 1
SOAP_ROUTER_MAX_EXPERTS = 1024
SOAP_ROUTER_MAX_TOP_K = 32

EXPORTED = [
    "soap_workspace_bytes", "soap_init_state", "soap_step", "soap_step_batched",
    "soap_last_error", "soap_qr_workspace_bytes", "soap_qr_f32", "soap_gemm_f32",
    "soap_factor_ema_f32", "soap_timing_enable", "soap_timing_num_stages",
    "soap_timing_stage_name", "soap_timing_collect", "soap_timing_reset", "soap_timing_get",
    "soap_kl_workspace_bytes", "soap_kl_step", "soap_kl_step_batched",
    "soap_kl_factors_workspace_bytes", "soap_kl_factors_f32", "soap_muon_workspace_bytes",
    "soap_muon_step", "soap_muon_step_batched", "soap_workspace_status",
    "soap_workspace_update_offset", "soap_test_force_qr_give_up", "soap_step_noalloc",
    "soap_test_qr_panel_path",
    "soap_layer_norm_forward", "soap_layer_norm_workspace_bytes", "soap_layer_norm_backward",
    "soap_router_rows", "soap_router_workspace_bytes", "soap_router_forward",
    "soap_router_backward", "soap_mx4_data_bytes", "soap_mx4_scale_bytes", "soap_mx4_quantize",
    "soap_mx4_gather", "soap_mx4_dequantize", "soap_mx4_gemm", "soap_mx4_gemm_rows", "soap_mx4_gemm_k",
]


class SoapError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"soap status {status}: {message}")
        self.status = status


_lib = None

_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_F = ctypes.c_float
_U32 = ctypes.c_uint32
_SZ = ctypes.c_size_t
_INT = ctypes.c_int


def lib() -> ctypes.CDLL:
    """Load the built library (build it with paper_2607_20548_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
    L = ctypes.CDLL(LIB_PATH)
    sig = {
        "soap_workspace_bytes": (_SZ, [_I64, _I64, _I64]),
        "soap_init_state": (_INT, [_I64, _I64, _I64, _P, _P, _P, _P, _P, _P, _P]),
        "soap_step": (_INT, [_P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _F, _F, _F, _F, _F,
                             _I64, _U32, _P, _SZ, _P]),
        "soap_step_batched": (_INT, [_I64, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _F, _F,
                                     _F, _F, _F, _I64, _U32, _P, _SZ, _P]),
        "soap_step_noalloc": (_INT, [_P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _F, _F, _F, _F,
                                     _F, _I64, _U32, _P]),
        "soap_kl_workspace_bytes": (_SZ, [_I64, _I64, _I64]),
        "soap_kl_step": (_INT, [_P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _F, _F, _F, _F, _F,
                                _F, _I64, _U32, _P, _SZ, _P]),
        "soap_kl_step_batched": (_INT, [_I64, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _F,
                                        _F, _F, _F, _F, _F, _I64, _U32, _P, _SZ, _P]),
        "soap_kl_factors_workspace_bytes": (_SZ, [_I64, _I64]),
        "soap_kl_factors_f32": (_INT, [_I64, _I64, _P, _P, _P, _P, _P, _F, _F, _P, _P, _P, _SZ,
                                       _P]),
        "soap_muon_workspace_bytes": (_SZ, [_I64, _I64, _I64]),
        "soap_muon_step": (_INT, [_P, _P, _P, _I64, _I64, _F, _F, _F, _F, _P, _I64, _U32, _P,
                                  _SZ, _P]),
        "soap_muon_step_batched": (_INT, [_I64, _P, _P, _P, _I64, _I64, _F, _F, _F, _F, _P, _I64,
                                          _U32, _P, _SZ, _P]),
        "soap_last_error": (ctypes.c_char_p, []),
        "soap_workspace_status": (_INT, [_P, ctypes.POINTER(ctypes.c_uint32), _P]),
        "soap_workspace_update_offset": (_SZ, [_I64, _I64, _I64]),
        "soap_test_force_qr_give_up": (_INT, [_U32]),
        "soap_test_qr_panel_path": (_INT, [_INT]),
        "soap_qr_workspace_bytes": (_SZ, [_I64]),
        "soap_qr_f32": (_INT, [_I64, _P, _P, _P, _P, _SZ, _P]),
        "soap_gemm_f32": (_INT, [_INT, _INT, _I64, _I64, _I64, _F, _P, _I64, _P, _I64, _F, _P,
                                 _I64, _P]),
        "soap_factor_ema_f32": (_INT, [_INT, _I64, _I64, _P, _P, _F, _P]),
        "soap_timing_enable": (_INT, [_INT]),
        "soap_timing_num_stages": (_INT, []),
        "soap_timing_stage_name": (ctypes.c_char_p, [_INT]),
        "soap_timing_collect": (_INT, []),
        "soap_timing_reset": (_INT, []),
        "soap_timing_get": (_INT, [_INT, ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_int64),
                                   ctypes.POINTER(ctypes.c_double)]),
        "soap_layer_norm_forward": (_INT, [_I64, _I64, _INT, _P, _I64, _P, _P, _F, _P, _I64, _P,
                                           _P, _P]),
        "soap_layer_norm_workspace_bytes": (_SZ, [_I64, _I64]),
        "soap_layer_norm_backward": (_INT, [_I64, _I64, _INT, _P, _I64, _P, _I64, _P, _P, _P, _P,
                                            _I64, _P, _P, _P, _SZ, _P]),
        "soap_router_rows": (_I64, [_I64, _I64, _I64]),
        "soap_router_workspace_bytes": (_SZ, [_I64, _I64]),
        "soap_router_forward": (_INT, [_I64, _I64, _I64, _INT, _P, _I64, _P, _U32, _F, _P, _P, _P,
                                       _P, _P, _P, _P, _P, _SZ, _P]),
        "soap_router_backward": (_INT, [_I64, _I64, _I64, _INT, _P, _I64, _P, _U32, _F, _P, _P,
                                        _P, _P, _P, _I64, _P]),
        "soap_mx4_data_bytes": (_SZ, [_I64, _I64]),
        "soap_mx4_scale_bytes": (_SZ, [_I64, _I64]),
        "soap_mx4_quantize": (_INT, [_I64, _I64, _I64, _INT, _P, _I64, _P, _I64, _P, _P, _P, _P,
                                     _P]),
        "soap_mx4_gather": (_INT, [_I64, _I64, _P, _I64, _P, _P, _P, _P, _P]),
        "soap_mx4_dequantize": (_INT, [_I64, _I64, _P, _P, _INT, _P, _I64, _P]),
        "soap_mx4_gemm": (_INT, [_I64, _I64, _I64, _P, _P, _P, _P, _INT, _P, _I64, _P]),
        "soap_mx4_gemm_rows": (_INT, [_I64, _I64, _I64, _I64, _P, _P, _P, _P, _P, _INT, _P, _I64,
                                      _P]),
        "soap_mx4_gemm_k": (_INT, [_I64, _I64, _I64, _I64, _P, _P, _P, _P, _P, _INT, _P, _P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    import torch
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"expected a torch tensor or an int pointer, got {type(x)}")
    if x.dtype != torch.float32 and x.dtype != torch.uint8:
        raise TypeError(f"tensors must be float32 (workspaces may be uint8), got {x.dtype}")
    if not x.is_cuda:
        raise ValueError("tensors must live on the GPU")
    if not x.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        if not torch.cuda.is_available():
            return None
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int) -> None:
    if status != SOAP_OK:
        raise SoapError(status, soap_last_error())


def soap_last_error() -> str:
    return lib().soap_last_error().decode()


def soap_workspace_bytes(batch: int, m: int, n: int) -> int:
    return lib().soap_workspace_bytes(batch, m, n)


def soap_workspace_status(workspace, stream=None):
    """Waits for the stream and returns (status code, status word) of the last
    step or QR enqueued with `workspace`: (SOAP_OK, 0) or
    (SOAP_ERR_QR_GAVE_UP, SOAP_STATUS_QR_* bits).  Other codes raise."""
    word = ctypes.c_uint32(0)
    rc = lib().soap_workspace_status(_ptr(workspace), ctypes.byref(word), _stream(stream))
    if rc not in (SOAP_OK, SOAP_ERR_QR_GAVE_UP):
        _check(rc)
    return rc, word.value


def soap_workspace_update_offset(batch: int, m: int, n: int) -> int:
    return lib().soap_workspace_update_offset(batch, m, n)


def soap_test_force_qr_give_up(mask: int) -> None:
    _check(lib().soap_test_force_qr_give_up(mask))


def soap_test_qr_panel_path(on: bool) -> None:
    _check(lib().soap_test_qr_panel_path(int(on)))


def soap_qr_workspace_bytes(n: int) -> int:
    return lib().soap_qr_workspace_bytes(n)


def soap_init_state(batch, m, n, L, R, Q_L, Q_R, M, V, stream=None) -> None:
    _check(lib().soap_init_state(batch, m, n, _ptr(L), _ptr(R), _ptr(Q_L), _ptr(Q_R), _ptr(M),
                                 _ptr(V), _stream(stream)))


def soap_step(param, grad, L, R, Q_L, Q_R, M, V, m, n, beta1, beta2, eps, lr, weight_decay,
              step, flags, workspace, workspace_bytes, stream=None) -> None:
    _check(lib().soap_step(_ptr(param), _ptr(grad), _ptr(L), _ptr(R), _ptr(Q_L), _ptr(Q_R),
                           _ptr(M), _ptr(V), m, n, beta1, beta2, eps, lr, weight_decay, step,
                           flags, _ptr(workspace), workspace_bytes, _stream(stream)))


SOAP_NOALLOC_MAX_WORKSPACE_BYTES = 256 << 20


def soap_step_noalloc(param, grad, L, R, Q_L, Q_R, M, V, m, n, beta1, beta2, eps, lr,
                      weight_decay, step, flags, stream=None) -> None:
    _check(lib().soap_step_noalloc(_ptr(param), _ptr(grad), _ptr(L), _ptr(R), _ptr(Q_L),
                                   _ptr(Q_R), _ptr(M), _ptr(V), m, n, beta1, beta2, eps, lr,
                                   weight_decay, step, flags, _stream(stream)))


def soap_step_batched(batch, param, grad, L, R, Q_L, Q_R, M, V, m, n, beta1, beta2, eps, lr,
                      weight_decay, step, flags, workspace, workspace_bytes, stream=None) -> None:
    _check(lib().soap_step_batched(batch, _ptr(param), _ptr(grad), _ptr(L), _ptr(R), _ptr(Q_L),
                                   _ptr(Q_R), _ptr(M), _ptr(V), m, n, beta1, beta2, eps, lr,
                                   weight_decay, step, flags, _ptr(workspace), workspace_bytes,
                                   _stream(stream)))


def soap_kl_workspace_bytes(batch: int, m: int, n: int) -> int:
    return lib().soap_kl_workspace_bytes(batch, m, n)


def soap_kl_step(param, grad, L, R, Q_L, Q_R, M, V, m, n, beta1, beta2, beta_kron, eps, lr,
                 weight_decay, step, flags, workspace, workspace_bytes, stream=None) -> None:
    _check(lib().soap_kl_step(_ptr(param), _ptr(grad), _ptr(L), _ptr(R), _ptr(Q_L), _ptr(Q_R),
                              _ptr(M), _ptr(V), m, n, beta1, beta2, beta_kron, eps, lr,
                              weight_decay, step, flags, _ptr(workspace), workspace_bytes,
                              _stream(stream)))


def soap_kl_step_batched(batch, param, grad, L, R, Q_L, Q_R, M, V, m, n, beta1, beta2, beta_kron,
                         eps, lr, weight_decay, step, flags, workspace, workspace_bytes,
                         stream=None) -> None:
    _check(lib().soap_kl_step_batched(batch, _ptr(param), _ptr(grad), _ptr(L), _ptr(R),
                                      _ptr(Q_L), _ptr(Q_R), _ptr(M), _ptr(V), m, n, beta1, beta2,
                                      beta_kron, eps, lr, weight_decay, step, flags,
                                      _ptr(workspace), workspace_bytes, _stream(stream)))


def soap_kl_factors_workspace_bytes(m: int, n: int) -> int:
    return lib().soap_kl_factors_workspace_bytes(m, n)


def soap_kl_factors_f32(m, n, G, L, R, Q_L, Q_R, beta_kron, eps, lam_L, lam_R, workspace,
                        workspace_bytes, stream=None) -> None:
    _check(lib().soap_kl_factors_f32(m, n, _ptr(G), _ptr(L), _ptr(R), _ptr(Q_L), _ptr(Q_R),
                                     beta_kron, eps, _ptr(lam_L), _ptr(lam_R), _ptr(workspace),
                                     workspace_bytes, _stream(stream)))


def _host_floats(values):
    """A host float array for a C `const float *` argument (kept alive by the caller)."""
    import numpy as np
    arr = np.ascontiguousarray(np.asarray(values, dtype=np.float32).ravel())
    return arr, arr.ctypes.data_as(ctypes.c_void_p)


def soap_muon_workspace_bytes(batch: int, m: int, n: int) -> int:
    return lib().soap_muon_workspace_bytes(batch, m, n)


def soap_muon_step(param, grad, M, m, n, beta1, lr, weight_decay, eps, coeffs, n_iters, flags,
                   workspace, workspace_bytes, stream=None) -> None:
    """coeffs: the 3 * n_iters Newton-Schulz coefficients (a_1, b_1, c_1, ...) on the host."""
    arr, ptr = _host_floats(coeffs)
    if arr.size < 3 * n_iters:
        raise ValueError("coeffs needs 3 * n_iters values")
    _check(lib().soap_muon_step(_ptr(param), _ptr(grad), _ptr(M), m, n, beta1, lr, weight_decay,
                                eps, ptr, n_iters, flags, _ptr(workspace), workspace_bytes,
                                _stream(stream)))


def soap_muon_step_batched(batch, param, grad, M, m, n, beta1, lr, weight_decay, eps, coeffs,
                           n_iters, flags, workspace, workspace_bytes, stream=None) -> None:
    arr, ptr = _host_floats(coeffs)
    if arr.size < 3 * n_iters:
        raise ValueError("coeffs needs 3 * n_iters values")
    _check(lib().soap_muon_step_batched(batch, _ptr(param), _ptr(grad), _ptr(M), m, n, beta1, lr,
                                        weight_decay, eps, ptr, n_iters, flags, _ptr(workspace),
                                        workspace_bytes, _stream(stream)))


def soap_qr_f32(n, A, Q, Rf, workspace, workspace_bytes, stream=None) -> None:
    _check(lib().soap_qr_f32(n, _ptr(A), _ptr(Q), _ptr(Rf), _ptr(workspace), workspace_bytes,
                             _stream(stream)))


def soap_gemm_f32(trans_a, trans_b, M, N, K, alpha, A, lda, B, ldb, beta, C, ldc,
                  stream=None) -> None:
    _check(lib().soap_gemm_f32(int(trans_a), int(trans_b), M, N, K, alpha, _ptr(A), lda, _ptr(B),
                               ldb, beta, _ptr(C), ldc, _stream(stream)))


def soap_factor_ema_f32(trans, m, n, G, F, beta, stream=None) -> None:
    _check(lib().soap_factor_ema_f32(int(trans), m, n, _ptr(G), _ptr(F), beta, _stream(stream)))


def soap_timing_enable(enable: bool) -> None:
    _check(lib().soap_timing_enable(int(bool(enable))))


def soap_timing_num_stages() -> int:
    return lib().soap_timing_num_stages()


def soap_timing_stage_name(stage: int) -> str:
    return lib().soap_timing_stage_name(stage).decode()


def soap_timing_collect() -> None:
    _check(lib().soap_timing_collect())


def soap_timing_reset() -> None:
    _check(lib().soap_timing_reset())


def soap_timing_get(stage: int):
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    fl = ctypes.c_double()
    _check(lib().soap_timing_get(stage, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl)))
    return ms.value, n.value, fl.value


# ---------------------------------------------------------------- helpers
class SoapState:
    """Device-resident SOAP state for `batch` m x n matrices (fp32, contiguous),
    allocated with torch and initialised by soap_init_state.  With ``kl`` the
    step is KL-SOAP (soap_kl_step), whose coefficient ``beta_kron`` step()
    then takes."""

    def __init__(self, m: int, n: int, batch: int = 1, device: str = "cuda", kl: bool = False):
        import torch
        self.m, self.n, self.batch = m, n, batch
        shp = (lambda r, c: (batch, r, c)) if batch > 1 else (lambda r, c: (r, c))
        kw = dict(dtype=torch.float32, device=device)
        self.L = torch.empty(shp(m, m), **kw)
        self.R = torch.empty(shp(n, n), **kw)
        self.Q_L = torch.empty(shp(m, m), **kw)
        self.Q_R = torch.empty(shp(n, n), **kw)
        self.M = torch.empty(shp(m, n), **kw)
        self.V = torch.empty(shp(m, n), **kw)
        self.kl = kl
        self.ws_bytes = (soap_kl_workspace_bytes if kl else soap_workspace_bytes)(batch, m, n)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        soap_init_state(batch, m, n, self.L, self.R, self.Q_L, self.Q_R, self.M, self.V)

    def status(self, stream=None):
        """(status code, SOAP_STATUS_QR_* bits) of the last step (synchronises)."""
        return soap_workspace_status(self.workspace, stream)

    def update(self):
        """The eigenbasis update N of the last step, a view into the workspace
        ([batch,] m x n fp32; valid until the next step)."""
        import torch
        off = soap_workspace_update_offset(self.batch, self.m, self.n)
        count = self.batch * self.m * self.n
        view = self.workspace[off:off + 4 * count].view(torch.float32)
        return view.view((self.batch, self.m, self.n) if self.batch > 1 else (self.m, self.n))

    def step(self, param, grad, t: int, beta1=0.95, beta2=0.95, eps=1e-8, lr=1e-3,
             weight_decay=0.1, flags=0, stream=None, beta_kron=None, refresh_every=1,
             stale_refresh=False) -> None:
        """One step t (1-based).  refresh_every = F refreshes the eigenbases
        when t mod F = 0 (SOAP_FLAG_SKIP_REFRESH on the other steps);
        stale_refresh sets SOAP_FLAG_STALE_REFRESH."""
        if refresh_every < 1:
            raise ValueError("refresh_every must be >= 1")
        if t % refresh_every != 0:
            flags |= SOAP_FLAG_SKIP_REFRESH
        if stale_refresh:
            flags |= SOAP_FLAG_STALE_REFRESH
        if self.kl:
            if beta_kron is None:
                raise ValueError("a KL-SOAP state needs beta_kron")
            if self.batch == 1:
                soap_kl_step(param, grad, self.L, self.R, self.Q_L, self.Q_R, self.M, self.V,
                             self.m, self.n, beta1, beta2, beta_kron, eps, lr, weight_decay, t,
                             flags, self.workspace, self.ws_bytes, stream)
            else:
                soap_kl_step_batched(self.batch, param, grad, self.L, self.R, self.Q_L, self.Q_R,
                                     self.M, self.V, self.m, self.n, beta1, beta2, beta_kron, eps,
                                     lr, weight_decay, t, flags, self.workspace, self.ws_bytes,
                                     stream)
            return
        if beta_kron is not None:
            raise ValueError("beta_kron applies to KL-SOAP states only")
        if self.batch == 1:
            soap_step(param, grad, self.L, self.R, self.Q_L, self.Q_R, self.M, self.V, self.m,
                      self.n, beta1, beta2, eps, lr, weight_decay, t, flags, self.workspace,
                      self.ws_bytes, stream)
        else:
            soap_step_batched(self.batch, param, grad, self.L, self.R, self.Q_L, self.Q_R, self.M,
                              self.V, self.m, self.n, beta1, beta2, eps, lr, weight_decay, t,
                              flags, self.workspace, self.ws_bytes, stream)


class MuonState:
    """Device-resident Muon state (the momentum buffer) for `batch` m x n
    matrices, zero-initialised, with its workspace."""

    def __init__(self, m: int, n: int, batch: int = 1, device: str = "cuda"):
        import torch
        self.m, self.n, self.batch = m, n, batch
        shp = (batch, m, n) if batch > 1 else (m, n)
        self.M = torch.zeros(shp, dtype=torch.float32, device=device)
        self.ws_bytes = soap_muon_workspace_bytes(batch, m, n)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    def step(self, param, grad, coeffs, beta1=0.9, lr=1e-3, weight_decay=0.1, eps=1e-7,
             bf16=False, stream=None) -> None:
        """coeffs: a sequence of (a, b, c) Newton-Schulz triples, one per iteration.
        bf16: Newton-Schulz in bfloat16 (SOAP_MUON_BF16)."""
        flat = [float(x) for abc in coeffs for x in abc]
        n_iters = len(flat) // 3
        flags = SOAP_MUON_BF16 if bf16 else 0
        if self.batch == 1:
            soap_muon_step(param, grad, self.M, self.m, self.n, beta1, lr, weight_decay, eps, flat,
                           n_iters, flags, self.workspace, self.ws_bytes, stream)
        else:
            soap_muon_step_batched(self.batch, param, grad, self.M, self.m, self.n, beta1, lr,
                                   weight_decay, eps, flat, n_iters, flags, self.workspace,
                                   self.ws_bytes, stream)


# ------------------------------------------------------------------------------
# Operators of the layer around an expert bank.  The functions of the C names take
# raw device pointers (ints) or tensors, whose element type and strides are the
# caller's to get right; the classes below check them.  None takes part in torch's
# autograd: results have no graph, the gradients are calls of their own.
def _raw(x) -> Optional[int]:
    if x is None or isinstance(x, int):
        return x
    if not x.is_cuda:
        raise ValueError("tensors must live on the GPU")
    return x.data_ptr()


def soap_layer_norm_forward(rows, cols, dtype, x, ldx, weight, bias, eps, y, ldy, mean, rstd,
                            stream=None) -> None:
    _check(lib().soap_layer_norm_forward(rows, cols, dtype, _raw(x), ldx, _raw(weight), _raw(bias),
                                         eps, _raw(y), ldy, _raw(mean), _raw(rstd),
                                         _stream(stream)))


def soap_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().soap_layer_norm_workspace_bytes(rows, cols))


def soap_layer_norm_backward(rows, cols, dtype, dy, lddy, x, ldx, weight, mean, rstd, dx, lddx,
                             dweight, dbias, workspace, workspace_bytes, stream=None) -> None:
    _check(lib().soap_layer_norm_backward(rows, cols, dtype, _raw(dy), lddy, _raw(x), ldx,
                                          _raw(weight), _raw(mean), _raw(rstd), _raw(dx), lddx,
                                          _raw(dweight), _raw(dbias), _raw(workspace),
                                          workspace_bytes, _stream(stream)))


def soap_router_rows(tokens: int, experts: int, top_k: int) -> int:
    return int(lib().soap_router_rows(tokens, experts, top_k))


def soap_router_workspace_bytes(tokens: int, experts: int) -> int:
    return int(lib().soap_router_workspace_bytes(tokens, experts))


def soap_router_forward(tokens, experts, top_k, dtype, logits, ld, token_mask, flags, balance, index,
                        gate, counts, loss, offsets, position, row_token, workspace, workspace_bytes,
                        stream=None) -> None:
    _check(lib().soap_router_forward(tokens, experts, top_k, dtype, _raw(logits), ld,
                                     _raw(token_mask), flags, balance, _raw(index), _raw(gate),
                                     _raw(counts), _raw(loss), _raw(offsets), _raw(position),
                                     _raw(row_token), _raw(workspace), workspace_bytes,
                                     _stream(stream)))


def soap_router_backward(tokens, experts, top_k, dtype, logits, ld, token_mask, flags, balance,
                         index, counts, dgate, dloss, dlogits, ldd, stream=None) -> None:
    _check(lib().soap_router_backward(tokens, experts, top_k, dtype, _raw(logits), ld,
                                      _raw(token_mask), flags, balance, _raw(index), _raw(counts),
                                      _raw(dgate), _raw(dloss), _raw(dlogits), ldd,
                                      _stream(stream)))


def soap_mx4_data_bytes(rows: int, k: int) -> int:
    return int(lib().soap_mx4_data_bytes(rows, k))


def soap_mx4_scale_bytes(rows: int, k: int) -> int:
    return int(lib().soap_mx4_scale_bytes(rows, k))


def soap_mx4_quantize(batch, rows, cols, dtype, x, ldx, row_index, x_rows, data, scale, data_t,
                      scale_t, stream=None) -> None:
    _check(lib().soap_mx4_quantize(batch, rows, cols, dtype, _raw(x), ldx, _raw(row_index), x_rows,
                                   _raw(data), _raw(scale), _raw(data_t), _raw(scale_t),
                                   _stream(stream)))


def soap_mx4_gather(rows, k, row_index, x_rows, x_data, x_scale, data, scale, stream=None) -> None:
    _check(lib().soap_mx4_gather(rows, k, _raw(row_index), x_rows, _raw(x_data), _raw(x_scale),
                                 _raw(data), _raw(scale), _stream(stream)))


def soap_mx4_dequantize(rows, k, data, scale, dtype, out, ldo, stream=None) -> None:
    _check(lib().soap_mx4_dequantize(rows, k, _raw(data), _raw(scale), dtype, _raw(out), ldo,
                                     _stream(stream)))


def soap_mx4_gemm(M, N, K, a_data, a_scale, b_data, b_scale, dtype, C, ldc, stream=None) -> None:
    _check(lib().soap_mx4_gemm(M, N, K, _raw(a_data), _raw(a_scale), _raw(b_data), _raw(b_scale),
                               dtype, _raw(C), ldc, _stream(stream)))


def soap_mx4_gemm_rows(groups, M, N, K, offsets, a_data, a_scale, b_data, b_scale, dtype, C, ldc,
                       stream=None) -> None:
    _check(lib().soap_mx4_gemm_rows(groups, M, N, K, _raw(offsets), _raw(a_data), _raw(a_scale),
                                    _raw(b_data), _raw(b_scale), dtype, _raw(C), ldc,
                                    _stream(stream)))


def soap_mx4_gemm_k(groups, M, N, K, offsets, a_data, a_scale, b_data, b_scale, dtype, C,
                    stream=None) -> None:
    _check(lib().soap_mx4_gemm_k(groups, M, N, K, _raw(offsets), _raw(a_data), _raw(a_scale),
                                 _raw(b_data), _raw(b_scale), dtype, _raw(C), _stream(stream)))


_torch = None


def _T():
    """torch, imported when a tensor is first needed."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _current_stream(t, name):
    """Raw current stream of the current device, where t must live."""
    T = _T()
    if not isinstance(t, T.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t)}")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must live on the GPU")
    if dev != T.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is "
                         f"cuda:{T.cuda.current_device()}")
    raw = getattr(T._C, "_cuda_getCurrentRawStream", None)
    return raw(dev) if raw is not None else T.cuda.current_stream().cuda_stream


def _floats(t, name, cols=None):
    """SOAP_F32 or SOAP_BF16 of a tensor of activations ([rows, cols] if cols is given)
    whose rows are contiguous."""
    T = _T()
    if cols is not None and (t.dim() != 2 or t.shape[1] != cols):
        raise ValueError(f"{name} must be [rows, {cols}], got {tuple(t.shape)}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    if t.dtype is T.bfloat16:
        return SOAP_BF16
    if t.dtype is T.float32:
        return SOAP_F32
    raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")


def _exactly(t, name, dtype, shape, like=None):
    """Checks a contiguous tensor of a given type and shape, on like's device (or, without
    one, on a GPU)."""
    T = _T()
    if not isinstance(t, T.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must live on the GPU")
    if like is not None and dev != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    return t


def _ld(t):
    """Row stride of a two-dimensional tensor (its width where it has at most one row)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _on(stream, inputs, call, *args, **kwargs):
    """call(...) on a stream of one's own: its outputs belong to that stream, and its
    inputs are kept from reuse until the stream has read them."""
    T = _T()
    inputs = [t for t in inputs if t is not None]
    for t in inputs:
        if not isinstance(t, T.Tensor):
            raise TypeError(f"expected a torch tensor, got {type(t)}")
        if t.get_device() < 0:
            raise ValueError("tensors must live on the GPU")
    if isinstance(stream, int):
        # the default stream's handle is 0, which ExternalStream takes for none given: it
        # would hand out a stream of its pool, that waits for nothing
        stream = T.cuda.ExternalStream(stream) if stream else T.cuda.default_stream()
    for t in inputs:
        t.record_stream(stream)
    with T.cuda.stream(stream):
        return call(*args, **kwargs)


class LayerNorm:
    """Layer norm of rows of `cols` values with fp32 ``weight`` and ``bias`` (either may
    be None): soap_layer_norm_forward / _backward with outputs and workspace allocated
    by torch.  Inputs are float32 or bfloat16 [rows, cols] with contiguous rows (other
    leading axes are the caller's to join); results have no autograd graph."""

    def __init__(self, weight=None, bias=None, eps: float = 1e-5, cols: Optional[int] = None):
        given = [t for t in (weight, bias) if t is not None]
        if cols is None:
            if not given:
                raise ValueError("a layer norm without weight and bias needs cols")
            cols = given[0].numel()
        for t, name in ((weight, "weight"), (bias, "bias")):
            if t is not None:
                _exactly(t, name, _T().float32, (cols,))
        self.weight, self.bias, self.eps, self.cols = weight, bias, eps, cols

    def _params(self, x):
        for t, name in ((self.weight, "weight"), (self.bias, "bias")):
            if t is not None and t.get_device() != x.get_device():
                raise ValueError(f"{name} is on {t.device}, not on {x.device}")

    def forward(self, x, stream=None):
        """(y, mean, rstd): y of x's type, the statistics float32 [rows]."""
        if stream is not None:
            return _on(stream, (x, self.weight, self.bias), self.forward, x)
        raw, kind, cols = _current_stream(x, "x"), _floats(x, "x", self.cols), self.cols
        self._params(x)
        rows, f32 = x.shape[0], _torch.float32
        y = x.new_empty((rows, cols))
        mean, rstd = x.new_empty(rows, dtype=f32), x.new_empty(rows, dtype=f32)
        w, b = self.weight, self.bias
        _check(lib().soap_layer_norm_forward(
            rows, cols, kind, x.data_ptr(), _ld(x), None if w is None else w.data_ptr(),
            None if b is None else b.data_ptr(), self.eps, y.data_ptr(), cols, mean.data_ptr(),
            rstd.data_ptr(), raw))
        return y, mean, rstd

    def backward(self, dy, x, mean, rstd, stream=None):
        """(dx, dweight, dbias); dweight and dbias are None without a weight and a bias."""
        if stream is not None:
            return _on(stream, (dy, x, mean, rstd, self.weight, self.bias), self.backward, dy, x, mean, rstd)
        raw, kind, cols = _current_stream(x, "x"), _floats(x, "x", self.cols), self.cols
        self._params(x)
        if dy.dtype is not x.dtype or dy.shape != x.shape or dy.get_device() != x.get_device():
            raise ValueError("dy must have x's type, shape and device")
        _floats(dy, "dy")
        rows, f32 = x.shape[0], _torch.float32
        _exactly(mean, "mean", f32, (rows,), x)
        _exactly(rstd, "rstd", f32, (rows,), x)
        L, w, b = lib(), self.weight, self.bias
        dx = x.new_empty((rows, cols))
        dweight = x.new_empty(cols, dtype=f32) if w is not None else None
        dbias = x.new_empty(cols, dtype=f32) if b is not None else None
        need = L.soap_layer_norm_workspace_bytes(rows, cols)
        work = x.new_empty(max(need, 16), dtype=_torch.uint8)
        _check(L.soap_layer_norm_backward(
            rows, cols, kind, dy.data_ptr(), _ld(dy), x.data_ptr(), _ld(x),
            None if w is None else w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), cols,
            None if w is None else dweight.data_ptr(), None if b is None else dbias.data_ptr(),
            work.data_ptr(), need, raw))
        return dx, dweight, dbias


class Routing:
    """What Router.forward found: index, gate [tokens, top_k], counts [experts + 1],
    loss [1] and the dispatch plan offsets [experts + 1], position [tokens, top_k],
    row_token [rows] (as soap_router_forward describes them)."""

    __slots__ = ("index", "gate", "counts", "loss", "offsets", "position", "row_token")


class Router:
    """Top-k routing over `experts` with balance loss, counts and dispatch plan
    (soap_router_forward / _backward).  Logits are float32 or bfloat16
    [tokens, experts] with contiguous rows, mask a bool [tokens] (False: the token
    does not route) or None; results have no autograd graph."""

    def __init__(self, experts: int, top_k: int, renormalize: bool = True, balance: float = 0.01):
        self.experts, self.top_k, self.balance = experts, top_k, balance
        self.flags = SOAP_ROUTER_RENORMALIZE if renormalize else 0

    def forward(self, logits, mask=None, stream=None) -> Routing:
        if stream is not None:
            return _on(stream, (logits, mask), self.forward, logits, mask)
        raw, kind = _current_stream(logits, "logits"), _floats(logits, "logits", self.experts)
        tokens, k, E = logits.shape[0], self.top_k, self.experts
        if mask is not None:
            _exactly(mask, "mask", _torch.bool, (tokens,), logits)
        L = lib()
        n, rows = tokens * k, L.soap_router_rows(tokens, E, k)
        need = L.soap_router_workspace_bytes(tokens, E)
        # one allocation of integers and one of floats, cut into the outputs
        ints = logits.new_empty(2 * n + 2 * (E + 1) + rows, dtype=_torch.int32)
        floats = logits.new_empty(n + 1, dtype=_torch.float32)
        work = logits.new_empty(max(need, 16), dtype=_torch.uint8)
        at, ft, c = ints.data_ptr(), floats.data_ptr(), 2 * n
        _check(L.soap_router_forward(
            tokens, E, k, kind, logits.data_ptr(), _ld(logits), None if mask is None else mask.data_ptr(),
            self.flags, self.balance, at, ft, at + 4 * c, ft + 4 * n, at + 4 * (c + E + 1), at + 4 * n,
            at + 4 * (c + 2 * (E + 1)), work.data_ptr(), need, raw))
        r = Routing()
        r.index = ints.as_strided((tokens, k), (k, 1), 0)
        r.position = ints.as_strided((tokens, k), (k, 1), n)
        r.counts = ints.as_strided((E + 1,), (1,), c)
        r.offsets = ints.as_strided((E + 1,), (1,), c + E + 1)
        r.row_token = ints.as_strided((rows,), (1,), c + 2 * (E + 1))
        r.gate = floats.as_strided((tokens, k), (k, 1), 0)
        r.loss = floats.as_strided((1,), (1,), n)
        return r

    def backward(self, logits, index, counts, dgate=None, dloss=None, mask=None, stream=None):
        """dlogits, of the logits' type, from the gradients of gate (float32
        [tokens, top_k]) and loss (float32 [1], None: 1)."""
        if stream is not None:
            return _on(stream, (logits, mask, index, counts, dgate, dloss), self.backward, logits, index,
                       counts, dgate, dloss, mask)
        raw, kind = _current_stream(logits, "logits"), _floats(logits, "logits", self.experts)
        tokens, k, E = logits.shape[0], self.top_k, self.experts
        i32, f32 = _torch.int32, _torch.float32
        if mask is not None:
            _exactly(mask, "mask", _torch.bool, (tokens,), logits)
        _exactly(index, "index", i32, (tokens, k), logits)
        _exactly(counts, "counts", i32, (E + 1,), logits)
        if dgate is not None:
            _exactly(dgate, "dgate", f32, (tokens, k), logits)
        if dloss is not None:
            _exactly(dloss, "dloss", f32, (1,), logits)
        out = logits.new_empty((tokens, E))
        _check(lib().soap_router_backward(
            tokens, E, k, kind, logits.data_ptr(), _ld(logits), None if mask is None else mask.data_ptr(),
            self.flags, self.balance, index.data_ptr(), counts.data_ptr(),
            None if dgate is None else dgate.data_ptr(), None if dloss is None else dloss.data_ptr(),
            out.data_ptr(), E, raw))
        return out


class Mx4:
    """A matrix, or a batch of them, in packed MXFP4 along its last axis of `k` values:
    ``data`` and ``scale`` uint8 [.., rows, bytes of a row]."""

    __slots__ = ("data", "scale", "k")

    def __init__(self, data, scale, k: int):
        u8, lead = _T().uint8, data.shape[:-1]
        padded = (k + 255) // 256 * 256
        _exactly(data, "data", u8, (*lead, padded // 2))
        _exactly(scale, "scale", u8, (*lead, padded // 32), data)
        if len(lead) not in (1, 2):
            raise ValueError("data must be [rows, bytes] or [batch, rows, bytes]")
        self.data, self.scale, self.k = data, scale, k

    @property
    def rows(self) -> int:
        return self.data.shape[-2]

    def values(self, dtype=None, stream=None):
        """What the packed values stand for, as float32 (default) or bfloat16 [.., rows, k]."""
        if stream is not None:
            return _on(stream, (self.data, self.scale), self.values, dtype)
        raw, kind, dtype = _current_stream(self.data, "data"), *_out_type(dtype)
        out = self.data.new_empty((*self.data.shape[:-1], self.k), dtype=dtype)
        if not self.k:
            return out
        _check(lib().soap_mx4_dequantize(out.numel() // self.k, self.k, self.data.data_ptr(),
                                         self.scale.data_ptr(), kind, out.data_ptr(), self.k, raw))
        return out


def _out_type(dtype):
    T = _T()
    if dtype is None or dtype is T.float32:
        return SOAP_F32, T.float32
    if dtype is T.bfloat16:
        return SOAP_BF16, dtype
    raise TypeError(f"results are float32 or bfloat16, not {dtype}")


def _mx4_empty(x, lead, k):
    """An Mx4 without contents, on x's device."""
    padded, u8 = (k + 255) // 256 * 256, _torch.uint8
    m = Mx4.__new__(Mx4)
    m.data, m.scale = x.new_empty((*lead, padded // 2), dtype=u8), x.new_empty((*lead, padded // 32), dtype=u8)
    m.k = k
    return m


def _taken_often(rows, x_rows, cols, kind):
    """Whether rows of x are quantised once and copied: two launches, which read a taken row
    packed, against one, which reads it whole and quantises it again (microseconds of the one
    / the other, rows of the plans of top-k routings to 64 experts).  The first costs a launch
    and a pass over x more, and saves by the values taken:
      bfloat16  4096 tokens of 2048: top 5 17.3 / 16.7, top 6 18.4 / 19.1, top 8 20.4 / 24.0
                4096 of 4096: top 2 16.3 / 15.3, top 3 18.5 / 20.7, top 8 29.6 / 48.2
                1024 of 2048: top 8 8.8 / 8.3, top 10 9.2 / 9.5
      float32   4096 of 2048: top 2 13.7 / 13.2, top 3 14.5 / 17.5, top 8 19.8 / 41.7
    A copied row keeps a wave busy from 2048 values on; rows of fewer win later (bfloat16, 32768
    tokens of 1024: top 3 39.0 / 36.5, top 4 45.3 / 47.1; 16384 of 768: top 8 37.2 / 37.1; 65536
    of 512: top 12 139 / 136).  Of 352 shapes (64 to 65536 tokens of 512 to 8192) it takes 0.3 per
    cent longer than the better form on average, 23 at worst.  Rows of -1 count, since the
    tokens are known on the GPU only: the worst are plans of mostly such rows (float32, 256 tokens
    of 4096, top 1 of 128 experts 7.7 / 6.6; 512 of 8192, top 2 of 64 11.9 / 9.7), of which others gain
    (64 of 4096, top 8 of 512 11.9 / 16.7)."""
    width = min((cols + 255) // 256 * 256, 1536)
    if kind == SOAP_BF16:
        return width > 512 and rows * cols * width >= ((28 << 20) + 1.6 * x_rows * cols) * 1536
    return width > 256 and rows * cols * width >= ((14 << 20) + 0.8 * x_rows * cols) * 1536


def mx4_quantize(x, along: str = "cols", row_index=None, stream=None):
    """x (float32 or bfloat16 [rows, cols], or contiguous [batch, rows, cols]) in MXFP4
    with blocks along its columns ("cols"), along its rows ("rows": the transposed
    matrix, [cols, rows]) or both (a pair, x read once).  row_index (int32 [n]) takes
    the rows row_index[i] of x, zeros where that is not a row of x; along the columns, rows
    that are taken often are quantised once into a packed matrix of x's own and copied."""
    if along not in ("cols", "rows", "both"):
        raise ValueError(f'along must be "cols", "rows" or "both", got {along!r}')
    if stream is not None:
        return _on(stream, (x, row_index), mx4_quantize, x, along, row_index)
    raw, kind, shape = _current_stream(x, "x"), _floats(x, "x"), x.shape
    if len(shape) not in (2, 3) or (len(shape) == 3 and not x.is_contiguous()):
        raise ValueError("x must be [rows, cols] or contiguous [batch, rows, cols]")
    cols, x_rows, lead = shape[-1], shape[-2], shape[:-2]
    rows = x_rows
    if row_index is not None:
        if lead:
            raise ValueError("row_index takes a single matrix")
        rows = row_index.numel()
        _exactly(row_index, "row_index", _torch.int32, (rows,), x)
    if row_index is not None and along == "cols" and _taken_often(rows, x_rows, cols, kind):
        once = mx4_quantize(x)
        a = _mx4_empty(x, (rows,), cols)
        _check(lib().soap_mx4_gather(rows, cols, row_index.data_ptr(), x_rows, once.data.data_ptr(),
                                     once.scale.data_ptr(), a.data.data_ptr(), a.scale.data_ptr(), raw))
        return a
    a = _mx4_empty(x, (*lead, rows), cols) if along != "rows" else None
    b = _mx4_empty(x, (*lead, cols), rows) if along != "cols" else None
    if rows and cols and 0 not in lead:        # there are values
        _check(lib().soap_mx4_quantize(
            lead[0] if lead else 1, rows, cols, kind, x.data_ptr(), cols if lead else _ld(x),
            None if row_index is None else row_index.data_ptr(), x_rows,
            None if a is None else a.data.data_ptr(), None if a is None else a.scale.data_ptr(),
            None if b is None else b.data.data_ptr(), None if b is None else b.scale.data_ptr(), raw))
    return (a, b) if along == "both" else a or b


def _mx4_check(a, b, dims_b):
    if a.data.dim() != 2 or b.data.dim() != dims_b:
        raise ValueError(f"a must be one matrix and b {'a batch' if dims_b == 3 else 'one matrix'}")
    if a.k != b.k:
        raise ValueError(f"a and b are summed over one axis: {a.k} and {b.k} values")
    if a.data.get_device() != b.data.get_device():
        raise ValueError(f"a is on {a.data.device}, b on {b.data.device}")


def mx4_product(a: Mx4, b: Mx4, dtype=None, stream=None):
    """a b^T, float32 (default) or bfloat16 [a.rows, b.rows] (soap_mx4_gemm)."""
    if stream is not None:
        return _on(stream, (a.data, a.scale, b.data, b.scale), mx4_product, a, b, dtype)
    _mx4_check(a, b, 2)
    raw, kind, dtype = _current_stream(a.data, "a"), *_out_type(dtype)
    out = a.data.new_empty((a.rows, b.rows), dtype=dtype)
    if not a.k or not out.numel():             # sums of nothing, or no sums
        return out.zero_()
    _check(lib().soap_mx4_gemm(a.rows, b.rows, a.k, a.data.data_ptr(), a.scale.data_ptr(),
                               b.data.data_ptr(), b.scale.data_ptr(), kind, out.data_ptr(), b.rows, raw))
    return out


def mx4_product_rows(a: Mx4, b: Mx4, offsets, dtype=None, stream=None):
    """Rows offsets[g] .. offsets[g + 1] of a times b[g]^T, [a.rows, b.rows]; zeros past the
    last group (soap_mx4_gemm_rows).  offsets: int32 [groups + 1] on the GPU."""
    if stream is not None:
        return _on(stream, (a.data, a.scale, b.data, b.scale, offsets), mx4_product_rows, a, b, offsets, dtype)
    _mx4_check(a, b, 3)
    raw, kind, dtype = _current_stream(a.data, "a"), *_out_type(dtype)
    groups = b.data.shape[0]
    _exactly(offsets, "offsets", _torch.int32, (groups + 1,), a.data)
    out = a.data.new_empty((a.rows, b.rows), dtype=dtype)
    if not a.k or not groups or not out.numel():
        return out.zero_()
    _check(lib().soap_mx4_gemm_rows(groups, a.rows, b.rows, a.k, offsets.data_ptr(), a.data.data_ptr(),
                                    a.scale.data_ptr(), b.data.data_ptr(), b.scale.data_ptr(), kind,
                                    out.data_ptr(), b.rows, raw))
    return out


def mx4_product_k(a: Mx4, b: Mx4, offsets, dtype=None, stream=None):
    """a b^T summed over k = offsets[g] .. offsets[g + 1] for every g, [groups, a.rows, b.rows]:
    the layout of the batched steps' gradients (soap_mx4_gemm_k)."""
    if stream is not None:
        return _on(stream, (a.data, a.scale, b.data, b.scale, offsets), mx4_product_k, a, b, offsets, dtype)
    _mx4_check(a, b, 2)
    raw, kind, dtype = _current_stream(a.data, "a"), *_out_type(dtype)
    _exactly(offsets, "offsets", _torch.int32, (offsets.numel(),), a.data)
    groups = offsets.numel() - 1
    if groups < 0:
        raise ValueError("offsets must hold at least one value")
    out = a.data.new_empty((groups, a.rows, b.rows), dtype=dtype)
    if not out.numel():
        return out
    _check(lib().soap_mx4_gemm_k(groups, a.rows, b.rows, a.k, offsets.data_ptr(), a.data.data_ptr(),
                                 a.scale.data_ptr(), b.data.data_ptr(), b.scale.data_ptr(), kind,
                                 out.data_ptr(), raw))
    return out
