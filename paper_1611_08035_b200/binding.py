"""ctypes binding of ``libb2gemm.so``: argument marshalling only.

Each Python function has the name and argument order of the C entry point it wraps (see
``include/b2gemm.h``); tensors are passed as raw device (or host) pointers plus sizes, the
stream as ``torch.cuda.current_stream().cuda_stream``.  No arithmetic of the GEMM happens
here.  Loading fails loudly when the library has not been built: there is no fallback.
"""
from __future__ import annotations

import ctypes
from ctypes import c_char, c_char_p, c_double, c_float, c_int, c_int64, c_size_t, c_void_p
from pathlib import Path

import torch

LIB_PATH = Path(__file__).resolve().parent / "libb2gemm.so"
_lib = None

_GEMM_TAIL_D = [c_char, c_char, c_int64, c_int64, c_int64, c_double, c_void_p, c_int64, c_void_p, c_int64, c_double,
                c_void_p, c_int64]
_GEMM_TAIL_S = [c_char, c_char, c_int64, c_int64, c_int64, c_float, c_void_p, c_int64, c_void_p, c_int64, c_float,
                c_void_p, c_int64]

_SIGNATURES = {
    "b2_dgemm": (c_int, _GEMM_TAIL_D + [c_void_p]),
    "b2_sgemm": (c_int, _GEMM_TAIL_S + [c_void_p]),
    "b2_dgemm_variant": (c_int, [c_int] + _GEMM_TAIL_D + [c_void_p]),
    "b2_sgemm_variant": (c_int, [c_int] + _GEMM_TAIL_S + [c_void_p]),
    "b2_device_status": (c_int, [c_void_p]),
    "b2_selftest_wait_timeout": (c_int, [c_void_p]),
    "b2_variant_count": (c_int, [c_int]),
    "b2_variant_name": (c_char_p, [c_int, c_int]),
    "b2_gemm_query_config": (c_int, [c_int, c_char, c_char, c_int64, c_int64, c_int64, c_int64, c_int64, c_int64,
                                     c_char_p, c_size_t]),
    "b2_zgemm4m_workspace_bytes": (c_size_t, [c_char, c_char, c_int64, c_int64, c_int64]),
    "b2_zgemm4m": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, ctypes.POINTER(c_double), c_void_p, c_int64,
                           c_void_p, c_int64, ctypes.POINTER(c_double), c_void_p, c_int64, c_void_p, c_size_t,
                           c_void_p]),
    "b2_dtrmm": (c_int, [c_char, c_char, c_char, c_char, c_int64, c_int64, c_double, c_void_p, c_int64, c_void_p, c_int64,
                         c_void_p]),
    "b2_strmm": (c_int, [c_char, c_char, c_char, c_char, c_int64, c_int64, c_float, c_void_p, c_int64, c_void_p, c_int64,
                         c_void_p]),
    "b2_dtrsm": (c_int, [c_char, c_char, c_char, c_char, c_int64, c_int64, c_double, c_void_p, c_int64, c_void_p, c_int64,
                         c_void_p]),
    "b2_strsm": (c_int, [c_char, c_char, c_char, c_char, c_int64, c_int64, c_float, c_void_p, c_int64, c_void_p, c_int64,
                         c_void_p]),
    "b2_gemm_splitk_auto": (c_int, [c_int64, c_int64, c_int64]),
    "b2_gemm_splitk_workspace_bytes": (c_size_t, [c_int, c_int64, c_int64, c_int64, c_int]),
    "b2_dgemm_splitk": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, c_double, c_void_p, c_int64, c_void_p, c_int64,
                                c_double, c_void_p, c_int64, c_int, c_void_p, c_size_t, c_void_p]),
    "b2_sgemm_splitk": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, c_float, c_void_p, c_int64, c_void_p, c_int64,
                                c_float, c_void_p, c_int64, c_int, c_void_p, c_size_t, c_void_p]),
    "b2_zgemm3m_workspace_bytes": (c_size_t, [c_char, c_char, c_int64, c_int64, c_int64]),
    "b2_zgemm3m": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, ctypes.POINTER(c_double), c_void_p, c_int64,
                           c_void_p, c_int64, ctypes.POINTER(c_double), c_void_p, c_int64, c_void_p, c_size_t,
                           c_void_p]),
    "b2_zgemm4m_static": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, ctypes.POINTER(c_double), c_void_p, c_int64,
                                  c_void_p, c_int64, ctypes.POINTER(c_double), c_void_p, c_int64, c_void_p]),
    "b2_dsyrk": (c_int, [c_char, c_char, c_int64, c_int64, c_double, c_void_p, c_int64, c_double, c_void_p, c_int64,
                         c_void_p]),
    "b2_ssyrk": (c_int, [c_char, c_char, c_int64, c_int64, c_float, c_void_p, c_int64, c_float, c_void_p, c_int64,
                         c_void_p]),
    "b2_dgemm_strided_batched": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, c_double, c_void_p, c_int64, c_int64,
                                         c_void_p, c_int64, c_int64, c_double, c_void_p, c_int64, c_int64, c_int64,
                                         c_void_p]),
    "b2_sgemm_strided_batched": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, c_float, c_void_p, c_int64, c_int64,
                                         c_void_p, c_int64, c_int64, c_float, c_void_p, c_int64, c_int64, c_int64,
                                         c_void_p]),
    "b2_sgemm_tf32_workspace_bytes": (c_size_t, [c_int, c_int64, c_int64, c_int64]),
    "b2_sgemm_tf32x1": (c_int, _GEMM_TAIL_S + [c_void_p, c_size_t, c_void_p]),
    "b2_sgemm_tf32x3": (c_int, _GEMM_TAIL_S + [c_void_p, c_size_t, c_void_p]),
    "b2_gemm_host_workspace_bytes": (c_size_t, [c_int, c_char, c_char, c_int64, c_int64, c_int64]),
    "b2_dgemm_host": (c_int, _GEMM_TAIL_D + [c_void_p, c_size_t, c_void_p]),
    "b2_sgemm_host": (c_int, _GEMM_TAIL_S + [c_void_p, c_size_t, c_void_p]),
    "b2_rmsnorm_f8": (c_int, [c_int64, c_int64, c_int, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_float, c_void_p,
                              c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p]),
    "b2_rmsnorm_backward_workspace_bytes": (c_size_t, [c_int64, c_int64]),
    "b2_rmsnorm_backward": (c_int, [c_int64, c_int64, c_int, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p,
                                    c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]),
    "b2_quant_f8": (c_int, [c_int64, c_int64, c_int, c_int, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64,
                            c_void_p]),
    "b2_gemm_f8_workspace_bytes": (c_size_t, [c_char, c_char, c_int64, c_int64, c_int64, c_void_p, c_int64, c_void_p,
                                              c_int64]),
    "b2_gemm_f8": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, c_float, c_void_p, c_int64, c_void_p, c_int64, c_int,
                           c_int, c_void_p, c_int64, c_void_p, c_int64, c_int, c_int, c_float, c_void_p, c_int64, c_int,
                           c_void_p, c_size_t, c_void_p]),
    "b2_wgrad_f8_workspace_bytes": (c_size_t, [c_int64, c_int64, c_int64, c_void_p, c_int64, c_void_p, c_int64]),
    "b2_wgrad_f8": (c_int, [c_int64, c_int64, c_int64, c_float, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64,
                            c_float, c_void_p, c_int64, c_int, c_void_p, c_size_t, c_void_p]),
    "b2_pipe_probe": (c_int, [c_int, c_int, c_int, c_int64, c_void_p, c_size_t, ctypes.POINTER(c_double), c_void_p]),
    "b2_model_throughput": (c_double, [c_int, ctypes.POINTER(c_double), ctypes.POINTER(c_double)]),
    "b2_model_stalled_throughput": (c_double, [c_double, c_int, c_double]),
    "b2_model_register_updates": (c_int, [c_int, c_int, c_int, c_int, c_int, c_int, ctypes.POINTER(c_int)]),
    "b2_model_predict_variant": (c_int, [c_int, c_int, ctypes.POINTER(c_double), c_char_p, c_size_t]),
    "b2_model_enumerate": (c_int, [c_int, c_int, c_char_p, c_size_t]),
    "b2_gemm_f8_act": (c_int, [c_char, c_char, c_int64, c_int64, c_int64, c_float] + 2 * [c_void_p, c_int64, c_void_p, c_int64, c_int, c_int]
                       + [c_int, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_int, c_void_p, c_int64, c_void_p, c_int64,
                          c_void_p, c_size_t, c_void_p]),
    "b2_act_backward_workspace_bytes": (c_size_t, [c_int64, c_int64]),
    "b2_act_backward": (c_int, [c_int64, c_int64, c_int, c_int] + 5 * [c_void_p, c_int64] + [c_void_p, c_void_p, c_size_t, c_void_p]),
    "b2_adamw": (c_int, [c_void_p, c_int] + 5 * [c_double] + [c_int64, ctypes.c_uint64, c_void_p, c_void_p, c_void_p, c_void_p]),
    "b2_graph_capture_id": (c_int, [c_void_p, ctypes.POINTER(ctypes.c_uint64)]),
    "b2_event_finish": (c_int, [c_void_p]),
    "b2_graph_watch": (c_int, [c_void_p, ctypes.POINTER(c_int)]),
    "b2_graph_gone": (c_int, [c_int]),
    "b2_graph_unwatch": (c_int, [c_int]),
    "b2_strerror": (c_char_p, [c_int]),
    "b2_version": (c_char_p, []),
}

EXPORTED_SYMBOLS = tuple(_SIGNATURES)


def lib() -> ctypes.CDLL:
    """The loaded C library (loaded once).  Raises when it has not been built."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1611_08035_b200.build` "
                "(there is no CPU or library fallback)")
        handle = ctypes.CDLL(str(LIB_PATH))
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
        _connect_calls(handle)
    return _lib


_connected: dict = {}  # name -> (address in the library, the function below) of what _b2calls was connected to


def _connect_calls(handle) -> None:
    """The 8-bit operators' functions below give way to those of ``_b2calls``, which read the same arguments without ctypes and fall
    back on these for keywords and for whatever they do not take.  Without that module these do all of it."""
    try:
        from . import _b2calls
    except ImportError:
        return
    names = ("b2_rmsnorm_f8", "b2_rmsnorm_backward", "b2_quant_f8", "b2_gemm_f8", "b2_wgrad_f8", "b2_gemm_f8_act", "b2_act_backward", "b2_adamw")
    table = {n: (ctypes.cast(getattr(handle, n), c_void_p).value, globals()[n]) for n in names}
    _b2calls.connect(B2Error, table)
    _connected.update(table)
    globals().update({n: getattr(_b2calls, n) for n in names})


def strerror(status: int) -> str:
    return lib().b2_strerror(int(status)).decode()


def version() -> str:
    return lib().b2_version().decode()


STATIC_LIMIT = 1005  # B2_ERR_STATIC_LIMIT


class B2Error(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} returned {status}: {strerror(status)}")
        self.status = status


_TR = {c: c.encode("ascii") for c in "NnTtCc"}


def _tr(c: str) -> bytes:
    b = _TR.get(c)
    return b if b is not None else c.encode("ascii")[:1]


# torch.cuda.current_stream() builds a Python Stream object (about 3 us per call, a third of the cost of
# launching a small GEMM from Python); the raw handle of the same stream comes from these two calls in 0.2 us.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream is not None and _cur_device is not None:
        return _raw_stream(_cur_device())
    return torch.cuda.current_stream().cuda_stream


def _check(fn: str, rc: int) -> None:
    if rc != 0:
        raise B2Error(fn, rc)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def b2_dgemm(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, variant=None, check=True) -> int:
    """C := alpha*op(A)*op(B) + beta*C in fp64 on device tensors (column-major storage)."""
    for t in (A, B, C):
        if t is not None and (t.dtype != torch.float64 or not t.is_cuda):
            raise TypeError("b2_dgemm takes float64 CUDA tensors")
    if variant is None:
        rc = lib().b2_dgemm(_tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb, beta, _ptr(C), ldc,
                            _stream())
    else:
        rc = lib().b2_dgemm_variant(variant, _tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb,
                                    beta, _ptr(C), ldc, _stream())
    if check:
        _check("b2_dgemm", rc)
    return rc


def b2_sgemm(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, variant=None, check=True) -> int:
    """C := alpha*op(A)*op(B) + beta*C in fp32 (FP32 FMA only) on device tensors."""
    for t in (A, B, C):
        if t is not None and (t.dtype != torch.float32 or not t.is_cuda):
            raise TypeError("b2_sgemm takes float32 CUDA tensors")
    if variant is None:
        rc = lib().b2_sgemm(_tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb, beta, _ptr(C), ldc,
                            _stream())
    else:
        rc = lib().b2_sgemm_variant(variant, _tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb,
                                    beta, _ptr(C), ldc, _stream())
    if check:
        _check("b2_sgemm", rc)
    return rc


def b2_variant_count(dtype: int) -> int:
    return lib().b2_variant_count(dtype)


def b2_variant_name(dtype: int, variant: int):
    s = lib().b2_variant_name(dtype, variant)
    return None if s is None else s.decode()


def b2_gemm_query_config(dtype, transa, transb, m, n, k, lda, ldb, ldc) -> str:
    buf = ctypes.create_string_buffer(1024)
    rc = lib().b2_gemm_query_config(dtype, _tr(transa), _tr(transb), m, n, k, lda, ldb, ldc, buf, len(buf))
    _check("b2_gemm_query_config", rc)
    return buf.value.decode()


def b2_zgemm4m_workspace_bytes(transa, transb, m, n, k) -> int:
    return lib().b2_zgemm4m_workspace_bytes(_tr(transa), _tr(transb), m, n, k)


def b2_zgemm4m(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    """Complex128 GEMM from four real-kernel launches; A, B, C complex128 CUDA tensors, workspace uint8."""
    for t in (A, B, C):
        if t is not None and (t.dtype != torch.complex128 or not t.is_cuda):
            raise TypeError("b2_zgemm4m takes complex128 CUDA tensors")
    al = (c_double * 2)(complex(alpha).real, complex(alpha).imag)
    be = (c_double * 2)(complex(beta).real, complex(beta).imag)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().b2_zgemm4m(_tr(transa), _tr(transb), m, n, k, al, _ptr(A), lda, _ptr(B), ldb, be, _ptr(C), ldc,
                          _ptr(workspace), wbytes, _stream())
    if check:
        _check("b2_zgemm4m", rc)
    return rc


def _tri(which, side, uplo, trans, diag, m, n, alpha, A, lda, B, ldb, check) -> int:
    dtype = next((t.dtype for t in (B, A) if t is not None), torch.float64)
    if dtype == torch.float64:
        name = f"b2_d{which}"
    elif dtype == torch.float32:
        name = f"b2_s{which}"
    else:
        raise TypeError(f"b2_{which} takes float64 or float32 tensors")
    for t in (A, B):
        if t is not None and (t.dtype != dtype or not t.is_cuda):
            raise TypeError(f"b2_{which} takes CUDA tensors of one dtype")
    rc = getattr(lib(), name)(_tr(side), _tr(uplo), _tr(trans), _tr(diag), m, n, alpha, _ptr(A), lda, _ptr(B), ldb,
                              _stream())
    if check:
        _check(name, rc)
    return rc


def b2_trmm(side, uplo, trans, diag, m, n, alpha, A, lda, B, ldb, check=True) -> int:
    """B := alpha*op(A)*B (side L) or alpha*B*op(A) (side R), A triangular; fp64 or fp32 by the tensors' dtype."""
    return _tri("trmm", side, uplo, trans, diag, m, n, alpha, A, lda, B, ldb, check)


def b2_trsm(side, uplo, trans, diag, m, n, alpha, A, lda, B, ldb, check=True) -> int:
    """Solve op(A)*X = alpha*B (side L) or X*op(A) = alpha*B (side R), A triangular; X overwrites B."""
    return _tri("trsm", side, uplo, trans, diag, m, n, alpha, A, lda, B, ldb, check)


def b2_gemm_splitk_auto(m, n, k) -> int:
    return lib().b2_gemm_splitk_auto(m, n, k)


def b2_gemm_splitk_workspace_bytes(dtype, m, n, k, splits=0) -> int:
    """dtype: torch.float64 / torch.float32."""
    return lib().b2_gemm_splitk_workspace_bytes(0 if dtype == torch.float64 else 1, m, n, k, splits)


def b2_gemm_splitk(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, splits=0, workspace=None,
                   check=True) -> int:
    """Split-K GEMM (fp64 or fp32 by the tensors' dtype); workspace: uint8 CUDA tensor or None."""
    if C.dtype == torch.float64:
        fn, name = lib().b2_dgemm_splitk, "b2_dgemm_splitk"
    elif C.dtype == torch.float32:
        fn, name = lib().b2_sgemm_splitk, "b2_sgemm_splitk"
    else:
        raise TypeError("b2_gemm_splitk takes float64 or float32 tensors")
    for t in (A, B, C):
        if t is not None and (t.dtype != C.dtype or not t.is_cuda):
            raise TypeError("b2_gemm_splitk takes CUDA tensors of one dtype")
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = fn(_tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb, beta, _ptr(C), ldc, splits,
            _ptr(workspace), wbytes, _stream())
    if check:
        _check(name, rc)
    return rc


def b2_zgemm3m_workspace_bytes(transa, transb, m, n, k) -> int:
    return lib().b2_zgemm3m_workspace_bytes(_tr(transa), _tr(transb), m, n, k)


def b2_zgemm3m(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    """Complex128 GEMM from three real-kernel launches (3M); same arguments as b2_zgemm4m."""
    for t in (A, B, C):
        if t is not None and (t.dtype != torch.complex128 or not t.is_cuda):
            raise TypeError("b2_zgemm3m takes complex128 CUDA tensors")
    al = (c_double * 2)(complex(alpha).real, complex(alpha).imag)
    be = (c_double * 2)(complex(beta).real, complex(beta).imag)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().b2_zgemm3m(_tr(transa), _tr(transb), m, n, k, al, _ptr(A), lda, _ptr(B), ldb, be, _ptr(C), ldc,
                          _ptr(workspace), wbytes, _stream())
    if check:
        _check("b2_zgemm3m", rc)
    return rc


ZGEMM4M_STATIC_BYTES = 6 << 20


def b2_zgemm4m_static(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, check=True) -> int:
    """b2_zgemm4m without a workspace argument, for callers that cannot allocate device memory.

    The scratch planes live in a ZGEMM4M_STATIC_BYTES array inside the library; problems that need more
    return B2_ERR_STATIC_LIMIT (1005).  Calls share that array: do not overlap them on the GPU."""
    for t in (A, B, C):
        if t is not None and (t.dtype != torch.complex128 or not t.is_cuda):
            raise TypeError("b2_zgemm4m_static takes complex128 CUDA tensors")
    al = (c_double * 2)(complex(alpha).real, complex(alpha).imag)
    be = (c_double * 2)(complex(beta).real, complex(beta).imag)
    rc = lib().b2_zgemm4m_static(_tr(transa), _tr(transb), m, n, k, al, _ptr(A), lda, _ptr(B), ldb, be, _ptr(C), ldc,
                                 _stream())
    if check:
        _check("b2_zgemm4m_static", rc)
    return rc


def b2_gemm_host_workspace_bytes(dtype, transa, transb, m, n, k) -> int:
    return lib().b2_gemm_host_workspace_bytes(dtype, _tr(transa), _tr(transb), m, n, k)


def _host_call(fn_name, want, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check):
    for t in (A, B, C):
        if t is not None and (t.dtype != want or t.is_cuda):
            raise TypeError(f"{fn_name} takes {want} HOST tensors")
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = getattr(lib(), fn_name)(_tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb, beta, _ptr(C),
                                 ldc, _ptr(workspace), wbytes, _stream())
    if check:
        _check(fn_name, rc)
    return rc


def b2_dgemm_host(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    """b2_dgemm on HOST tensors (pinned for speed); copies in, computes on the GPU, copies C back."""
    return _host_call("b2_dgemm_host", torch.float64, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc,
                      workspace, check)


def b2_sgemm_host(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    """b2_sgemm on HOST tensors (pinned for speed); copies in, computes on the GPU, copies C back."""
    return _host_call("b2_sgemm_host", torch.float32, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc,
                      workspace, check)


def b2_model_throughput(rates, jobs) -> float:
    """Section 4: outer products per cycle of an instruction mix = min over pipelines of rate/jobs."""
    n = len(rates)
    if n != len(jobs):
        raise ValueError("rates and jobs must have the same length")
    r = (c_double * max(n, 1))(*rates)
    j = (c_double * max(n, 1))(*jobs)
    return lib().b2_model_throughput(n, r, j)


def b2_model_stalled_throughput(jobs: float, n_dependent: int, latency: float) -> float:
    return lib().b2_model_stalled_throughput(jobs, n_dependent, latency)


def b2_model_register_updates(r_total, mr, nr, v, r_a, r_r) -> int:
    """Section 5: floor((R_total - mr*nr/v - R_A) / R_R)."""
    out = c_int(0)
    _check("b2_model_register_updates", lib().b2_model_register_updates(r_total, mr, nr, v, r_a, r_r, ctypes.byref(out)))
    return out.value


def b2_model_enumerate(dtype: int, top: int = 16) -> str:
    """Ranked candidate micro-kernels/tiles of the pipeline model as a JSON string (host-only call)."""
    buf = ctypes.create_string_buffer(1 << 16)
    _check("b2_model_enumerate", lib().b2_model_enumerate(dtype, top, buf, len(buf)))
    return buf.value.decode()


def b2_model_predict_variant(dtype: int, variant: int):
    """(predicted fraction of pipe peak, JSON description) of a kernel variant from the pipeline model."""
    frac = c_double(0.0)
    buf = ctypes.create_string_buffer(1024)
    _check("b2_model_predict_variant", lib().b2_model_predict_variant(dtype, variant, ctypes.byref(frac), buf, len(buf)))
    return frac.value, buf.value.decode()


def b2_device_status() -> int:
    """Synchronise the current stream and return (and clear) the device status word: 0 or B2_ERR_TIMEOUT."""
    return lib().b2_device_status(_stream())


def b2_selftest_wait_timeout() -> int:
    """Enqueue the bounded-wait self-test kernel (the next b2_device_status then reports B2_ERR_TIMEOUT)."""
    return lib().b2_selftest_wait_timeout(_stream())


def b2_sgemm_tf32_workspace_bytes(terms: int, m: int, n: int, k: int) -> int:
    return lib().b2_sgemm_tf32_workspace_bytes(terms, m, n, k)


def b2_sgemm_tf32(terms, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    """fp32 GEMM on the tensor cores in TF32 (terms=1: b2_sgemm_tf32x1, terms=3: b2_sgemm_tf32x3); device tensors."""
    for t in (A, B, C):
        if t is not None and (t.dtype != torch.float32 or not t.is_cuda):
            raise TypeError("b2_sgemm_tf32 takes float32 CUDA tensors")
    fn = {1: lib().b2_sgemm_tf32x1, 3: lib().b2_sgemm_tf32x3}[terms]
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = fn(_tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, _ptr(B), ldb, beta, _ptr(C), ldc, _ptr(workspace),
            wbytes, _stream())
    if check:
        _check(f"b2_sgemm_tf32x{terms}", rc)
    return rc


def b2_sgemm_tf32x1(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    return b2_sgemm_tf32(1, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check)


def b2_sgemm_tf32x3(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check=True) -> int:
    return b2_sgemm_tf32(3, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, workspace, check)


def b2_syrk(uplo, trans, n, k, alpha, A, lda, beta, C, ldc, check=True) -> int:
    """Symmetric rank-k update on the uplo triangle of C (b2_dsyrk / b2_ssyrk by dtype); device tensors."""
    if C is not None and C.dtype == torch.float32:
        fn, name = lib().b2_ssyrk, "b2_ssyrk"
    else:
        fn, name = lib().b2_dsyrk, "b2_dsyrk"
    for t in (A, C):
        if t is not None and (not t.is_cuda or (C is not None and t.dtype != C.dtype)):
            raise TypeError(f"{name} takes CUDA tensors of one dtype")
    rc = fn(_tr(uplo), _tr(trans), n, k, alpha, _ptr(A), lda, beta, _ptr(C), ldc, _stream())
    if check:
        _check(name, rc)
    return rc


def b2_gemm_strided_batched(transa, transb, m, n, k, alpha, A, lda, stride_a, B, ldb, stride_b, beta, C, ldc, stride_c,
                            batch, check=True) -> int:
    """`batch` GEMMs of one shape on strided operands (b2_dgemm_strided_batched / b2_sgemm_strided_batched)."""
    if C is not None and C.dtype == torch.float32:
        fn, name = lib().b2_sgemm_strided_batched, "b2_sgemm_strided_batched"
    else:
        fn, name = lib().b2_dgemm_strided_batched, "b2_dgemm_strided_batched"
    for t in (A, B, C):
        if t is not None and (not t.is_cuda or (C is not None and t.dtype != C.dtype)):
            raise TypeError(f"{name} takes CUDA tensors of one dtype")
    rc = fn(_tr(transa), _tr(transb), m, n, k, alpha, _ptr(A), lda, stride_a, _ptr(B), ldb, stride_b, beta, _ptr(C), ldc,
            stride_c, batch, _stream())
    if check:
        _check(name, rc)
    return rc


# ---- linear layers in 8 bits --------------------------------------------------------------------------------
# A decoding step makes these calls on a few tokens, where the GPU needs two or three microseconds: once the library is loaded
# the functions of csrc/calls.cpp take their place (norm of 8 tokens: 8.3 us a call here, of which ctypes takes 1.5, 5 there).
_TYPES = {torch.float32: 1, torch.bfloat16: 2}  # B2_TYPE_*
_SCALES = {torch.float8_e8m0fnu: 0, torch.float32: 1}  # B2_SCALE_*
_E4M3, _E8M0, _F32, _BF16 = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float32, torch.bfloat16


def _refuse(fn: str, *args) -> None:
    """args: (name, tensor or None, allowed dtypes).  Raises for the first one that is not a CUDA tensor of such a type."""
    for name, t, allowed in args:
        if t is not None and (t.dtype not in allowed or not t.is_cuda):
            raise TypeError(f"{fn}: {name} is {t.dtype} on {t.device}; it takes a CUDA tensor of {' or '.join(map(str, allowed))}")
    raise TypeError(f"{fn}: tensors of different types")


def b2_rmsnorm_f8(d, t, x, ldx, residual, ldr, w, eps, h, ldh, q, ldq, s, lds, rstd, check=True) -> int:
    """h = x + residual; y = h / sqrt(mean(h^2) + eps) * w per token (column of d); y leaves as e4m3 numbers q with e8m0
    scales s, one for 128 features.  x, residual, w, h: bfloat16 or float32 alike; residual, h and rstd (float32) may be None."""
    dt = x.dtype
    if not (dt in _TYPES and w.dtype is dt and q.dtype is _E4M3 and s.dtype is _E8M0 and x.is_cuda and w.is_cuda and q.is_cuda and s.is_cuda
            and (residual is None or (residual.dtype is dt and residual.is_cuda)) and (h is None or (h.dtype is dt and h.is_cuda))
            and (rstd is None or (rstd.dtype is _F32 and rstd.is_cuda))):
        _refuse("b2_rmsnorm_f8", ("x", x, tuple(_TYPES)), ("residual", residual, (dt,)), ("w", w, (dt,)), ("h", h, (dt,)), ("q", q, (_E4M3,)),
                ("s", s, (_E8M0,)), ("rstd", rstd, (_F32,)))
    rc = (_lib or lib()).b2_rmsnorm_f8(d, t, _TYPES[dt], x.data_ptr(), ldx, None if residual is None else residual.data_ptr(), ldr, w.data_ptr(),
                                       eps, None if h is None else h.data_ptr(), ldh, q.data_ptr(), ldq, s.data_ptr(), lds,
                                       None if rstd is None else rstd.data_ptr(), _stream())
    if rc and check:
        raise B2Error("b2_rmsnorm_f8", rc)
    return rc


def b2_rmsnorm_backward_workspace_bytes(d: int, t: int) -> int:
    return lib().b2_rmsnorm_backward_workspace_bytes(d, t)


def b2_rmsnorm_backward(d, t, dy, lddy, h, ldh, rstd, w, dh, lddh, dx, lddx, dw, workspace, check=True) -> int:
    """Gradients of the norm: dx (of x and residual alike; dh, the gradient that reaches h directly, is added, or None)
    and dw (float32, d).  dy, h, w, dh, dx: bfloat16 or float32 alike."""
    dt = dy.dtype
    if not (dt in _TYPES and h.dtype is dt and w.dtype is dt and dx.dtype is dt and rstd.dtype is _F32 and dw.dtype is _F32 and dy.is_cuda
            and h.is_cuda and w.is_cuda and dx.is_cuda and rstd.is_cuda and dw.is_cuda and (dh is None or (dh.dtype is dt and dh.is_cuda))
            and (workspace is None or workspace.is_cuda)):
        _refuse("b2_rmsnorm_backward", ("dy", dy, tuple(_TYPES)), ("h", h, (dt,)), ("w", w, (dt,)), ("dh", dh, (dt,)), ("dx", dx, (dt,)),
                ("rstd", rstd, (_F32,)), ("dw", dw, (_F32,)), ("workspace", workspace, (torch.uint8,)))
    rc = (_lib or lib()).b2_rmsnorm_backward(d, t, _TYPES[dt], dy.data_ptr(), lddy, h.data_ptr(), ldh, rstd.data_ptr(), w.data_ptr(),
                                             None if dh is None else dh.data_ptr(), lddh, dx.data_ptr(), lddx, dw.data_ptr(),
                                             None if workspace is None else workspace.data_ptr(),
                                             0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    if rc and check:
        raise B2Error("b2_rmsnorm_backward", rc)
    return rc


def b2_quant_f8(d, t, block, x, ldx, q, ldq, s, lds, check=True) -> int:
    """x (d x t, bfloat16 or float32) as e4m3 numbers q with e8m0 scales s for blocks of 128 features by 1 or 128 tokens."""
    code = _TYPES.get(x.dtype)
    if not (code and q.dtype is _E4M3 and s.dtype is _E8M0 and x.is_cuda and q.is_cuda and s.is_cuda):
        _refuse("b2_quant_f8", ("x", x, tuple(_TYPES)), ("q", q, (_E4M3,)), ("s", s, (_E8M0,)))
    rc = (_lib or lib()).b2_quant_f8(d, t, block, code, x.data_ptr(), ldx, q.data_ptr(), ldq, s.data_ptr(), lds, _stream())
    if rc and check:
        raise B2Error("b2_quant_f8", rc)
    return rc


def b2_gemm_f8_workspace_bytes(transa, transb, m, n, k, A, lda, B, ldb) -> int:
    return lib().b2_gemm_f8_workspace_bytes(_tr(transa), _tr(transb), m, n, k, _ptr(A), lda, _ptr(B), ldb)


def b2_gemm_f8(transa, transb, m, n, k, alpha, A, lda, SA, ldsa, block_a, B, ldb, SB, ldsb, block_b, beta, C, ldc,
               workspace=None, check=True) -> int:
    """C := alpha*op(A)*op(B) + beta*C of block-scaled e4m3 matrices; scales float8_e8m0fnu or float32, C bfloat16 or float32."""
    code, ca, cb = _TYPES.get(C.dtype), _SCALES.get(SA.dtype), _SCALES.get(SB.dtype)
    if not (code and ca is not None and cb is not None and A.dtype is _E4M3 and B.dtype is _E4M3 and A.is_cuda and B.is_cuda and C.is_cuda
            and SA.is_cuda and SB.is_cuda and (workspace is None or workspace.is_cuda)):
        _refuse("b2_gemm_f8", ("A", A, (_E4M3,)), ("SA", SA, tuple(_SCALES)), ("B", B, (_E4M3,)), ("SB", SB, tuple(_SCALES)),
                ("C", C, tuple(_TYPES)), ("workspace", workspace, (torch.uint8,)))
    rc = (_lib or lib()).b2_gemm_f8(_tr(transa), _tr(transb), m, n, k, alpha, A.data_ptr(), lda, SA.data_ptr(), ldsa, block_a, ca, B.data_ptr(), ldb,
                                    SB.data_ptr(), ldsb, block_b, cb, beta, C.data_ptr(), ldc, code,
                                    None if workspace is None else workspace.data_ptr(),
                                    0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    if rc and check:
        raise B2Error("b2_gemm_f8", rc)
    return rc


def b2_wgrad_f8_workspace_bytes(m, n, k, Q, ldq, Y, ldy) -> int:
    return lib().b2_wgrad_f8_workspace_bytes(m, n, k, _ptr(Q), ldq, _ptr(Y), ldy)


def b2_wgrad_f8(m, n, k, alpha, Q, ldq, S, lds, Y, ldy, beta, C, ldc, workspace=None, check=True) -> int:
    """C (m x n) := alpha * X Y^T + beta*C over k tokens, X = Q*S an activation kept in 8 bits, Y bfloat16 gradients."""
    code = _TYPES.get(C.dtype)
    if not (code and Q.dtype is _E4M3 and S.dtype is _E8M0 and Y.dtype is _BF16 and Q.is_cuda and S.is_cuda and Y.is_cuda and C.is_cuda
            and (workspace is None or workspace.is_cuda)):
        _refuse("b2_wgrad_f8", ("Q", Q, (_E4M3,)), ("S", S, (_E8M0,)), ("Y", Y, (_BF16,)), ("C", C, tuple(_TYPES)),
                ("workspace", workspace, (torch.uint8,)))
    rc = (_lib or lib()).b2_wgrad_f8(m, n, k, alpha, Q.data_ptr(), ldq, S.data_ptr(), lds, Y.data_ptr(), ldy, beta, C.data_ptr(), ldc, code,
                                     None if workspace is None else workspace.data_ptr(),
                                     0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    if rc and check:
        raise B2Error("b2_wgrad_f8", rc)
    return rc


ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU, ACT_GRADIENT = 0, 1, 2, 3, 4, 16  # B2_ACT_*


def b2_gemm_f8_act(transa, transb, m, n, k, alpha, A, lda, SA, ldsa, block_a, B, ldb, SB, ldsb, block_b, act, bias, z, ldz, residual, ldr, c, ldc,
                   q, ldq, s, lds, workspace=None, check=True) -> int:
    """z = alpha*op(A)*op(B) + bias, c = act(z) + residual of block-scaled e4m3 matrices; or, with act | ACT_GRADIENT, c = alpha*op(A)*op(B) * act'(z) +
    residual with z given.  z, residual, c: bfloat16 or float32 alike; q, s: c as e4m3 numbers with e8m0 scales; bias: float32.  bias, z, residual,
    c or q (with s) may be None.  The workspace is b2_gemm_f8_workspace_bytes'."""
    dt = next((t.dtype for t in (c, z, residual) if t is not None), _F32)
    code, ca, cb = _TYPES.get(dt), _SCALES.get(SA.dtype), _SCALES.get(SB.dtype)
    if not (code and ca is not None and cb is not None and A.dtype is _E4M3 and B.dtype is _E4M3 and A.is_cuda and B.is_cuda and SA.is_cuda and SB.is_cuda
            and all(t is None or (t.dtype is dt and t.is_cuda) for t in (z, residual, c)) and (bias is None or (bias.dtype is _F32 and bias.is_cuda))
            and (q is None or (q.dtype is _E4M3 and q.is_cuda)) and (s is None or (s.dtype is _E8M0 and s.is_cuda)) and (workspace is None or workspace.is_cuda)):
        _refuse("b2_gemm_f8_act", ("A", A, (_E4M3,)), ("SA", SA, tuple(_SCALES)), ("B", B, (_E4M3,)), ("SB", SB, tuple(_SCALES)), ("bias", bias, (_F32,)),
                ("c", c, tuple(_TYPES)), ("z", z, (dt,) if code else tuple(_TYPES)), ("residual", residual, (dt,) if code else tuple(_TYPES)), ("q", q, (_E4M3,)),
                ("s", s, (_E8M0,)), ("workspace", workspace, (torch.uint8,)))
    rc = (_lib or lib()).b2_gemm_f8_act(_tr(transa), _tr(transb), m, n, k, alpha, A.data_ptr(), lda, SA.data_ptr(), ldsa, block_a, ca, B.data_ptr(), ldb,
                                        SB.data_ptr(), ldsb, block_b, cb, act, _ptr(bias) or None, _ptr(z) or None, ldz, _ptr(residual) or None, ldr,
                                        _ptr(c) or None, ldc, code, _ptr(q) or None, ldq, _ptr(s) or None, lds, _ptr(workspace) or None,
                                        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    if rc and check:
        raise B2Error("b2_gemm_f8_act", rc)
    return rc


def b2_act_backward_workspace_bytes(d: int, t: int) -> int:
    return lib().b2_act_backward_workspace_bytes(d, t)


def b2_act_backward(d, t, act, dy, lddy, z, ldz, dz, lddz, q, ldq, s, lds, db, workspace=None, check=True) -> int:
    """dz = dy * act'(z) and db = its sum over the tokens, dz also as e4m3 numbers q with e8m0 scales s.  dy, z, dz: bfloat16 or float32 alike; db: float32.
    z may be None with ACT_NONE; dz, q (with s) and db where they are not wanted."""
    dt = dy.dtype
    if not (dt in _TYPES and dy.is_cuda and all(x is None or (x.dtype is dt and x.is_cuda) for x in (z, dz)) and (q is None or (q.dtype is _E4M3 and q.is_cuda))
            and (s is None or (s.dtype is _E8M0 and s.is_cuda)) and (db is None or (db.dtype is _F32 and db.is_cuda)) and (workspace is None or workspace.is_cuda)):
        _refuse("b2_act_backward", ("dy", dy, tuple(_TYPES)), ("z", z, (dt,)), ("dz", dz, (dt,)), ("q", q, (_E4M3,)), ("s", s, (_E8M0,)), ("db", db, (_F32,)),
                ("workspace", workspace, (torch.uint8,)))
    rc = (_lib or lib()).b2_act_backward(d, t, _TYPES[dt], act, dy.data_ptr(), lddy, _ptr(z) or None, ldz, _ptr(dz) or None, lddz, _ptr(q) or None, ldq,
                                         _ptr(s) or None, lds, _ptr(db) or None, _ptr(workspace) or None,
                                         0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    if rc and check:
        raise B2Error("b2_act_backward", rc)
    return rc


class _AdamwTensor(ctypes.Structure):  # b2_adamw_tensor
    _fields_ = [(f, c_void_p) for f in ("param", "grad", "m", "v", "sm", "sv")] + [("n", c_int64), ("type_param", ctypes.c_int32), ("type_grad", ctypes.c_int32),
                                                                                 ("state_bits", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def b2_adamw(params, grads, m, v, sm, sv, lr, beta1, beta2, eps, weight_decay, step, seed=0, grad_scale=None, check=True) -> int:
    """One AdamW step, in place, over lists of contiguous tensors of one device, the current one.  params, grads: bfloat16 or float32; m, v: float32, or float8_e4m3fn (v then holds the root of the
    second moment) with float8_e8m0fnu scales sm, sv for 128 elements each.  sm and sv may be None, as may their entries for float32 states.  lr and
    step are numbers, or CUDA tensors of one float32 and one int64 that are read when the call runs; grad_scale: a CUDA tensor of one float32, or None."""
    count = len(params)
    if any(len(x) != count for x in (grads, m, v)) or any(x is not None and len(x) != count for x in (sm, sv)):
        raise ValueError("b2_adamw: the lists have different lengths")
    devices = {x.device for some in (params, grads, m, v, sm or (), sv or (), (lr, step, grad_scale)) for x in some if getattr(x, "is_cuda", False)}
    if len(devices) > 1:
        raise ValueError(f"b2_adamw: the tensors of a call are on one device; these are on {sorted(map(str, devices))}")
    table = (_AdamwTensor * max(count, 1))()
    for i in range(count):
        t = (params[i], grads[i], m[i], v[i], None if sm is None else sm[i], None if sv is None else sv[i])
        n, bits = t[0].numel(), 8 if t[2].dtype is _E4M3 else 32
        state = (_E4M3,) if bits == 8 else (_F32,)
        kinds = (tuple(_TYPES), tuple(_TYPES), state, state)
        if not all(x.is_cuda and x.dtype in k for x, k in zip(t, kinds)):
            _refuse(f"b2_adamw: tensor {i}", *zip(("param", "grad", "m", "v"), t, kinds))
        if not all(x.is_contiguous() and x.numel() == n for x in t[:4]):
            raise ValueError(f"b2_adamw: tensor {i}: param, grad, m and v are contiguous and of one size; they have {[tuple(x.shape) for x in t[:4]]}")
        if bits == 8:
            for x in t[4:]:
                if x is None or not x.is_cuda or x.dtype is not _E8M0 or not x.is_contiguous() or x.numel() != (n + 127) // 128:
                    raise ValueError(f"b2_adamw: tensor {i}: states in 8 bits have contiguous float8_e8m0fnu scales, {(n + 127) // 128} of them")
        table[i] = _AdamwTensor(*[_ptr(x) or None for x in t[:4]], *([_ptr(x) or None for x in t[4:]] if bits == 8 else (None, None)), n, _TYPES[t[0].dtype],
                                _TYPES[t[1].dtype], bits, 0)
    on_device = []
    for name, x, dt in (("lr", lr, _F32), ("step", step, torch.int64), ("grad_scale", grad_scale, _F32)):
        if isinstance(x, torch.Tensor) and (not x.is_cuda or x.dtype is not dt or x.numel() != 1):
            raise TypeError(f"b2_adamw: {name} is {x.dtype} {tuple(x.shape)} on {x.device}; as a tensor it is one {dt} on a CUDA device")
        on_device.append(x.data_ptr() if isinstance(x, torch.Tensor) else None)
    rc = (_lib or lib()).b2_adamw(table, count, 0.0 if on_device[0] else lr, beta1, beta2, eps, weight_decay, 1 if on_device[1] else step, seed & 0xFFFFFFFFFFFFFFFF,
                                  on_device[2], on_device[0], on_device[1], _stream())
    if rc and check:
        raise B2Error("b2_adamw", rc)
    return rc


def b2_graph_capture_id(stream: int) -> int:
    """The number of the capture that a stream (its handle) is in; 0 where it is in none."""
    number = ctypes.c_uint64()
    rc = lib().b2_graph_capture_id(stream, ctypes.byref(number))
    if rc:
        raise B2Error("b2_graph_capture_id", rc)
    return number.value


def b2_event_finish(event: int) -> None:
    """Waits on the host for an event (its handle) of no capture, also in the middle of one."""
    rc = lib().b2_event_finish(event)
    if rc:
        raise B2Error("b2_event_finish", rc)


def b2_graph_watch(stream: int) -> int:
    """A watch of the graph that a stream (its handle) is captured into."""
    watch = c_int()
    rc = lib().b2_graph_watch(stream, ctypes.byref(watch))
    if rc:
        raise B2Error("b2_graph_watch", rc)
    return watch.value


def b2_graph_gone(watch: int) -> bool:
    return bool(lib().b2_graph_gone(watch))


def b2_graph_unwatch(watch: int) -> None:
    rc = lib().b2_graph_unwatch(watch)
    if rc:
        raise B2Error("b2_graph_unwatch", rc)
