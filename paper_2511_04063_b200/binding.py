"""ctypes binding of the C ABI declared in include/dartquant.h.

Argument marshalling only: every step of the calibration path runs in the CUDA
kernels of libdartquant.so.  PyTorch supplies device memory and streams.  There
is no fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdartquant.so")

DQ_OK, DQ_ERR_INVALID_ARG, DQ_ERR_UNSUPPORTED, DQ_ERR_ALLOC, DQ_ERR_CUDA = 0, 1, 2, 3, 4
DQ_ERR_SINGULAR, DQ_ERR_NONFINITE, DQ_ERR_TIMEOUT, DQ_ERR_NOT_CONVERGED = 5, 6, 7, 8
DQ_QR_HOUSEHOLDER, DQ_QR_ITERATIVE = 0, 1
DQ_ORTH_QR, DQ_ORTH_CAYLEY = 0, 1
DQ_OBJ_WHIP, DQ_OBJ_VARIANCE, DQ_OBJ_KURTOSIS, DQ_OBJ_QUANT = 0, 1, 2, 3
DQ_FP32, DQ_BF16, DQ_FP16 = 0, 1, 2
DQ_MXFP4, DQ_MXFP8 = 0, 1
DQ_QK_NORM, DQ_QK_NEIGHBOURS, DQ_QK_HADAMARD = 1, 2, 4
DQ_PATH_FP32, DQ_PATH_BF16_TC = 0, 1
DQ_MEAN_TOKENS, DQ_SUM_TOKENS = 0, 1
DQ_SGD, DQ_SGD_MOMENTUM, DQ_ADAM = 0, 1, 2
DQ_PHASE_NAMES = ("qr_forward", "rotate_whip", "grad_rotation", "qr_backward", "update")
DQ_BUF_R, DQ_BUF_U, DQ_BUF_GQ, DQ_BUF_GZ, DQ_BUF_G, DQ_BUF_PARTIALS, DQ_BUF_Z, DQ_BUF_OPT_M, DQ_BUF_OPT_V = range(9)
DQ_BUF_CAYLEY_M, DQ_BUF_CAYLEY_ALPHA = 9, 10

EXPORTED_SYMBOLS = (
    "dq_calib_init", "dq_calib_step", "dq_calib_get_rotation", "dq_rotate_apply",
    "dq_calib_get_latent", "dq_calib_set_latent", "dq_calib_refresh_inputs", "dq_calib_status",
    "dq_calib_get_timings", "dq_calib_set_timing", "dq_calib_debug_buffer", "dq_calib_launch_count", "dq_status_string",
    "dq_calib_destroy", "dq_version", "dq_rotate_apply_static", "dq_calib_set_qr_method", "dq_calib_set_optimizer", "dq_gather_tokens", "dq_eval_rotation",
    "dq_calib_set_orth_method", "dq_calib_set_objective", "dq_calib_run_epochs", "dq_calib_mma_flops", "dq_calib_set_keep_gradient",
    "dq_calib_set_backward_precision", "dq_calib_selftest_bounded_wait", "dq_calib_time_product",
    "dq_mx_row_bytes", "dq_mx_scale_bytes", "dq_mx_linear_workspace", "dq_mx_quantize", "dq_mx_dequantize", "dq_rmsnorm_quantize",
    "dq_mx_matmul", "dq_mx_linear", "dq_mx_status", "dq_mx_selftest_bounded_wait",
    "dq_kv_page_bytes", "dq_kv_attention_workspace", "dq_kv_evict_workspace", "dq_qk_norm_rope", "dq_kv_append", "dq_kv_dequantize",
    "dq_kv_attention", "dq_kv_attention_weights", "dq_kv_evict",
)


class dq_calib_config(C.Structure):
    _fields_ = [("d", C.c_int32), ("n_tokens", C.c_int64), ("batch", C.c_int32), ("x_dtype", C.c_int32),
                ("path", C.c_int32), ("reduction", C.c_int32), ("optimizer", C.c_int32), ("lr", C.c_float),
                ("ldx", C.c_int64)]


class dq_heads_t(C.Structure):
    _fields_ = [("d_data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("heads", C.c_int32)]


class dq_kv_cache_t(C.Structure):
    _fields_ = [("d_pages", C.c_void_p), ("n_pages", C.c_int64), ("d_table", C.c_void_p), ("d_lengths", C.c_void_p),
                ("n_seqs", C.c_int32), ("table_width", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32)]


class DartQuantError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (dq_status %d)" % (where, status_string(status), status))


_lib = None


def load_library(path: str = LIB_PATH) -> C.CDLL:
    """Loads libdartquant.so.  Raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError("libdartquant.so is not built: run `python -m paper_2511_04063_b200.build` "
                          "(the calibration path has no non-CUDA implementation)")
    lib = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    lib.dq_calib_init.argtypes = [C.POINTER(vp), C.POINTER(dq_calib_config), vp, vp, vp]
    lib.dq_calib_step.argtypes = [vp, i32, vp]
    lib.dq_calib_get_rotation.argtypes = [vp, vp]
    lib.dq_rotate_apply.argtypes = [vp, i32, i64, i32, i64, vp, vp, i64, vp]
    lib.dq_rotate_apply_static.argtypes = [vp, i64, i32, i64, vp, vp, i64, vp]
    lib.dq_rotate_apply_static.restype = i32
    lib.dq_calib_set_optimizer.argtypes = [vp, i32, C.c_float, C.c_float, C.c_float, C.c_float]
    lib.dq_calib_set_optimizer.restype = i32
    lib.dq_calib_set_qr_method.argtypes = [vp, i32, i32]
    lib.dq_calib_set_qr_method.restype = i32
    lib.dq_calib_run_epochs.argtypes = [vp, vp, i64, i64, C.c_float, i32, i32, C.c_uint64, vp, C.POINTER(i64)]
    lib.dq_calib_run_epochs.restype = i32
    lib.dq_calib_set_objective.argtypes = [vp, i32, i32]
    lib.dq_calib_set_objective.restype = i32
    lib.dq_calib_set_orth_method.argtypes = [vp, i32, C.c_float, C.c_float, i32]
    lib.dq_calib_set_orth_method.restype = i32
    lib.dq_gather_tokens.argtypes = [vp, i32, i64, i32, i64, C.c_uint64, i64, i64, vp, i64, vp]
    lib.dq_gather_tokens.restype = i32
    lib.dq_eval_rotation.argtypes = [vp, i32, i64, i32, i64, vp, C.c_float, i32, vp, vp]
    lib.dq_eval_rotation.restype = i32
    lib.dq_calib_get_latent.argtypes = [vp, vp]
    lib.dq_calib_set_latent.argtypes = [vp, vp]
    lib.dq_calib_status.argtypes = [vp]
    lib.dq_calib_refresh_inputs.argtypes = [vp]
    lib.dq_calib_get_timings.argtypes = [vp, C.POINTER(C.c_float), i32]
    lib.dq_calib_set_timing.argtypes = [vp, i32]
    lib.dq_calib_debug_buffer.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(i64)]
    lib.dq_calib_set_keep_gradient.argtypes = [vp, i32]
    lib.dq_calib_set_keep_gradient.restype = i32
    lib.dq_calib_selftest_bounded_wait.argtypes = [vp, C.c_uint64, vp]
    lib.dq_calib_selftest_bounded_wait.restype = i32
    lib.dq_calib_time_product.argtypes = [vp, i32, i32, C.POINTER(C.c_float)]
    lib.dq_calib_time_product.restype = i32
    lib.dq_calib_set_backward_precision.argtypes = [vp, i32]
    lib.dq_calib_set_backward_precision.restype = i32
    heads, cache = C.POINTER(dq_heads_t), C.POINTER(dq_kv_cache_t)
    for name, args in (("dq_mx_quantize", [vp, i32, i64, i64, i64, i32, vp, vp, vp, i64, vp]),
                       ("dq_mx_dequantize", [i32, vp, vp, i64, i64, vp, i32, i64, vp]),
                       ("dq_rmsnorm_quantize", [vp, vp, i32, i64, i64, i64, i64, vp, i32, C.c_float, i32, vp, vp, vp, i64, vp, i64,
                                                vp]),
                       ("dq_mx_matmul", [i32, vp, vp, i64, vp, vp, i64, i64, vp, i32, i64, vp]),
                       ("dq_mx_linear", [vp, i32, i64, i64, i64, i32, vp, vp, i64, vp, i32, i64, vp, vp]),
                       ("dq_mx_selftest_bounded_wait", [i32, vp, vp, i64, vp, vp, i64, i64, vp, i32, i64, i64, C.c_uint64, vp]),
                       ("dq_mx_status", [vp]),
                       ("dq_qk_norm_rope", [heads, heads, i32, i64, i32, vp, vp, i32, vp, vp, i32, C.c_float, i32, heads, heads, vp]),
                       ("dq_kv_append", [heads, heads, i32, i64, cache, vp, heads, heads, vp, vp, i64, vp]),
                       ("dq_kv_dequantize", [cache, vp, i64, heads, heads, i32, vp]),
                       ("dq_kv_attention", [heads, i32, i64, cache, vp, C.c_float, heads, vp, vp, vp]),
                       ("dq_kv_attention_weights", [heads, i32, i64, vp, cache, vp, C.c_float, vp, vp, i64, vp]),
                       ("dq_kv_evict", [cache, vp, vp, i64, i32, i32, vp, vp, vp, vp, vp])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i32
    for name, args in (("dq_mx_row_bytes", [i32, i64]), ("dq_mx_scale_bytes", [i64, i64]),
                       ("dq_mx_linear_workspace", [i32, i64, i64]), ("dq_kv_page_bytes", [i32, i32]),
                       ("dq_kv_attention_workspace", [i32]), ("dq_kv_evict_workspace", [i32, i32, i32])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i64
    lib.dq_calib_launch_count.argtypes = [vp]
    lib.dq_calib_mma_flops.argtypes = [vp]
    lib.dq_calib_mma_flops.restype = C.c_double
    lib.dq_calib_launch_count.restype = i64
    lib.dq_status_string.argtypes = [i32]
    lib.dq_status_string.restype = C.c_char_p
    lib.dq_calib_destroy.argtypes = [vp]
    lib.dq_calib_destroy.restype = None
    lib.dq_version.restype = C.c_char_p
    for name in ("dq_calib_init", "dq_calib_step", "dq_calib_get_rotation", "dq_rotate_apply",
                 "dq_calib_get_latent", "dq_calib_set_latent", "dq_calib_status", "dq_calib_get_timings",
                 "dq_calib_set_timing", "dq_calib_debug_buffer", "dq_calib_refresh_inputs"):
        getattr(lib, name).restype = i32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().dq_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != DQ_OK:
        raise DartQuantError(status, where)


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


def _stream_ptr(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


# ---------------------------------------------------------------------------
# Same-name wrappers (torch tensors in, raw pointers out)
# ---------------------------------------------------------------------------
def dq_calib_init(X, Z0, *, lr: float, path: int, reduction: int = DQ_MEAN_TOKENS, stream=None):
    """X: CUDA tensor [batch, N, d] or [N, d], float32 or bfloat16, contiguous rows (borrowed:
    keep it alive).  Z0: CUDA float32 [batch, d, d] or [d, d] (copied).  Returns an opaque handle."""
    import torch
    assert X.is_cuda and Z0.is_cuda and Z0.dtype == torch.float32 and Z0.is_contiguous()
    if X.dim() == 2:
        X = X.unsqueeze(0)
    batch, n, d = X.shape
    assert X.stride(2) == 1 and X.stride(0) == n * X.stride(1)
    cfg = dq_calib_config(d=d, n_tokens=n, batch=batch,
                          x_dtype=DQ_FP32 if X.dtype == torch.float32 else DQ_BF16, path=path,
                          reduction=reduction, optimizer=DQ_SGD, lr=lr, ldx=X.stride(1))
    h = C.c_void_p(0)
    _check(load_library().dq_calib_init(C.byref(h), C.byref(cfg), _ptr(X), _ptr(Z0), _stream_ptr(stream)),
           "dq_calib_init")
    return h


def dq_calib_step(h, n_steps: int, loss_out=None):
    _check(load_library().dq_calib_step(h, n_steps, _ptr(loss_out)), "dq_calib_step")


def dq_calib_get_rotation(h, R_out):
    _check(load_library().dq_calib_get_rotation(h, _ptr(R_out)), "dq_calib_get_rotation")


def dq_calib_get_latent(h, Z_out):
    _check(load_library().dq_calib_get_latent(h, _ptr(Z_out)), "dq_calib_get_latent")


def dq_calib_set_latent(h, Z):
    _check(load_library().dq_calib_set_latent(h, _ptr(Z)), "dq_calib_set_latent")


def dq_calib_refresh_inputs(h):
    _check(load_library().dq_calib_refresh_inputs(h), "dq_calib_refresh_inputs")


def dq_calib_status(h) -> int:
    return int(load_library().dq_calib_status(h))


def dq_calib_set_timing(h, enabled: bool):
    _check(load_library().dq_calib_set_timing(h, int(enabled)), "dq_calib_set_timing")


def dq_calib_set_optimizer(h, optimizer: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8):
    _check(load_library().dq_calib_set_optimizer(h, optimizer, lr, beta1, beta2, eps), "dq_calib_set_optimizer")


def dq_calib_set_qr_method(h, method: int, n_iters: int = 0):
    _check(load_library().dq_calib_set_qr_method(h, method, n_iters), "dq_calib_set_qr_method")


def dq_calib_run_epochs(h, pool, sample_ratio: float, accum: int, n_epochs: int, seed: int, loss_out=None) -> int:
    """pool: CUDA tensor [n_pool, d] (row stride = pool.stride(0)).  Returns the number of optimiser steps."""
    steps = C.c_int64(0)
    _check(load_library().dq_calib_run_epochs(h, pool.data_ptr(), pool.shape[0], pool.stride(0), sample_ratio, accum,
                                              n_epochs, seed, loss_out.data_ptr() if loss_out is not None else None,
                                              C.byref(steps)), "dq_calib_run_epochs")
    return int(steps.value)


def dq_calib_set_keep_gradient(h, keep: bool = True):
    _check(load_library().dq_calib_set_keep_gradient(h, 1 if keep else 0), "dq_calib_set_keep_gradient")


def dq_calib_set_backward_precision(h, split: bool):
    """QR-Orth backward on split-bf16 operands (True) or plain bf16 operands (False, the default)."""
    _check(load_library().dq_calib_set_backward_precision(h, 1 if split else 0), "dq_calib_set_backward_precision")


def dq_calib_selftest_bounded_wait(h, limit_ns: int) -> int:
    """Runs the library's bounded in-kernel wait on a barrier nothing arrives at; returns the nanoseconds it
    waited before giving up (synchronises).  Leaves DQ_ERR_TIMEOUT in the handle's status word."""
    import torch
    waited = torch.zeros(1, dtype=torch.int64, device="cuda")
    _check(load_library().dq_calib_selftest_bounded_wait(h, limit_ns, waited.data_ptr()), "dq_calib_selftest_bounded_wait")
    return int(waited.cpu()[0])


def dq_calib_time_product(h, nterms: int, reps: int = 10) -> float:
    """Mean milliseconds of one dense d^3 QR-Orth product (nterms 3: split-bf16, 1: plain bf16); measurement."""
    ms = C.c_float(0.0)
    _check(load_library().dq_calib_time_product(h, nterms, reps, C.byref(ms)), "dq_calib_time_product")
    return float(ms.value)


def dq_calib_mma_flops(h) -> float:
    return float(load_library().dq_calib_mma_flops(h))


def dq_calib_set_objective(h, objective: int, bits: int = 0):
    _check(load_library().dq_calib_set_objective(h, objective, bits), "dq_calib_set_objective")


def dq_calib_set_orth_method(h, method: int, beta: float = 0.0, q: float = 0.0, s: int = 0):
    _check(load_library().dq_calib_set_orth_method(h, method, beta, q, s), "dq_calib_set_orth_method")


def dq_calib_get_timings(h) -> dict:
    arr = (C.c_float * len(DQ_PHASE_NAMES))()
    _check(load_library().dq_calib_get_timings(h, arr, len(DQ_PHASE_NAMES)), "dq_calib_get_timings")
    return {k: float(arr[i]) for i, k in enumerate(DQ_PHASE_NAMES)}


def dq_calib_debug_buffer(h, which: int, dtype, shape):
    """A torch view (no copy) of one of the handle's device workspaces."""
    import torch
    p, n = C.c_void_p(0), C.c_int64(0)
    _check(load_library().dq_calib_debug_buffer(h, which, C.byref(p), C.byref(n)), "dq_calib_debug_buffer")
    numel = 1
    for s in shape:
        numel *= s
    assert numel <= n.value, (numel, n.value)
    itemsize = torch.empty((), dtype=dtype).element_size()
    buf = (C.c_byte * (numel * itemsize)).from_address(p.value)
    # wrap device memory through the CUDA array interface
    class _Wrap:
        pass
    w = _Wrap()
    typestr = {torch.float32: "<f4", torch.bfloat16: "<i2"}[dtype]
    w.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (p.value, False),
                                  "version": 2}
    del buf
    t = torch.as_tensor(w, device="cuda")
    return t.view(torch.bfloat16) if dtype == torch.bfloat16 else t


def dq_calib_launch_count(h) -> int:
    return int(load_library().dq_calib_launch_count(h))


def dq_calib_destroy(h):
    load_library().dq_calib_destroy(h)


def dq_rotate_apply(X, R, Y, stream=None):
    """Y = X R.  X, Y: CUDA [n, d] float32 or bfloat16 (same dtype); R: CUDA float32 [d, d]."""
    import torch
    assert X.is_cuda and R.is_cuda and Y.is_cuda and X.dtype == Y.dtype and R.dtype == torch.float32
    assert X.stride(1) == 1 and Y.stride(1) == 1 and R.is_contiguous()
    n, d = X.shape
    _check(load_library().dq_rotate_apply(_ptr(X), DQ_FP32 if X.dtype == torch.float32 else DQ_BF16, n, d,
                                          X.stride(0), _ptr(R), _ptr(Y), Y.stride(0), _stream_ptr(stream)),
           "dq_rotate_apply")


def dq_rotate_apply_static(X, R, Y, stream=None):
    """Y = X R for bfloat16 X, Y ([n, d]) and float32 R ([d, d]) without any device allocation:
    for callers whose memory is all spoken for (see include/dartquant.h).  d <= 2048."""
    import torch
    assert X.is_cuda and R.is_cuda and Y.is_cuda and R.dtype == torch.float32
    assert X.dtype == torch.bfloat16 and Y.dtype == torch.bfloat16
    assert X.stride(1) == 1 and Y.stride(1) == 1 and R.is_contiguous()
    n, d = X.shape
    _check(load_library().dq_rotate_apply_static(_ptr(X), n, d, X.stride(0), _ptr(R), _ptr(Y), Y.stride(0),
                                                 _stream_ptr(stream)), "dq_rotate_apply_static")


def dq_gather_tokens(X, seed: int, first: int, count: int, out, stream=None):
    """out[i] = X[pi_seed(first + i)]: seeded sampling of token rows without replacement.
    X: CUDA [n, d] float32 or bfloat16; out: CUDA [count, d] of the same dtype."""
    import torch
    assert X.is_cuda and out.is_cuda and X.dtype == out.dtype and X.dim() == 2 and out.dim() == 2
    n, d = X.shape
    _check(load_library().dq_gather_tokens(_ptr(X), DQ_FP32 if X.dtype == torch.float32 else DQ_BF16, n, d,
                                           X.stride(0), seed, first, count, _ptr(out), out.stride(0),
                                           _stream_ptr(stream)), "dq_gather_tokens")


def dq_eval_rotation(X, R, tau: float, bits: int, stream=None):
    """(number of outliers |o| > tau, mean squared per-token asymmetric quantisation error) of O = X R.
    X: CUDA [n, d] float32 or bfloat16; R: CUDA float32 [d, d].  Synchronises to read the result."""
    import torch
    assert X.is_cuda and R.is_cuda and R.dtype == torch.float32 and X.dim() == 2
    assert X.stride(1) == 1 and R.is_contiguous()
    n, d = X.shape
    out = torch.zeros(2, dtype=torch.float64, device=X.device)
    _check(load_library().dq_eval_rotation(_ptr(X), DQ_FP32 if X.dtype == torch.float32 else DQ_BF16, n, d,
                                           X.stride(0), _ptr(R), tau, bits, _ptr(out), _stream_ptr(stream)),
           "dq_eval_rotation")
    res = out.cpu()
    return int(round(float(res[0]))), float(res[1])


# ---------------------------------------------------------------------------
# Microscaled operators.  Their arguments are checked and passed on by the compiled module _calls (csrc/py_calls.cpp): a
# ctypes call with checks in Python takes longer than the smaller kernels.  A wrong tensor raises ValueError, a refusal of
# the library DartQuantError.
# ---------------------------------------------------------------------------
_calls = None


def _mx():
    """The compiled calls, bound to the library."""
    global _calls
    if _calls is None:
        import torch
        lib = load_library()
        try:
            from . import _calls as calls
        except ImportError as e:
            raise ImportError("the microscaled and key/value cache operators' Python calls are not built for this interpreter: run "
                              "`python -m paper_2511_04063_b200.build` where its Python.h is installed") from e
        torch.cuda.current_device()
        calls.bind(tuple(C.cast(getattr(lib, n), C.c_void_p).value for n in
                         ("dq_mx_quantize", "dq_mx_dequantize", "dq_rmsnorm_quantize", "dq_mx_matmul", "dq_mx_linear")),
                   (torch.float32, torch.bfloat16, torch.float16), torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
        calls.bind_kv(tuple(C.cast(getattr(lib, n), C.c_void_p).value for n in
                            ("dq_qk_norm_rope", "dq_kv_append", "dq_kv_dequantize", "dq_kv_attention", "dq_kv_attention_weights",
                             "dq_kv_evict", "dq_kv_attention_workspace", "dq_kv_evict_workspace")), torch.int32)
        _calls = calls
    return _calls


def dq_mx_row_bytes(fmt: int, k: int) -> int:
    return int(load_library().dq_mx_row_bytes(fmt, k))


def dq_mx_scale_bytes(rows: int, k: int) -> int:
    return int(load_library().dq_mx_scale_bytes(rows, k))


def dq_mx_linear_workspace(a_fmt: int, m: int, k: int) -> int:
    return int(load_library().dq_mx_linear_workspace(a_fmt, m, k))


def dq_mx_empty(rows: int, k: int, fmt: int, device="cuda"):
    """(codes, scales): buffers for a [rows, k] matrix, torch.uint8."""
    import torch
    if fmt != DQ_MXFP4 and fmt != DQ_MXFP8:
        raise ValueError("format %r: DQ_MXFP4 or DQ_MXFP8 is needed" % (fmt,))
    return (torch.empty((rows, dq_mx_row_bytes(fmt, k)), dtype=torch.uint8, device=device),
            torch.empty(dq_mx_scale_bytes(rows, k), dtype=torch.uint8, device=device))


def dq_mx_quantize(X, fmt: int, codes, scales, values=None, stream=None):
    """Codes and scales of X ([rows, k]; float32, bfloat16 or float16).  values (same type and shape; may be X): what
    the codes stand for."""
    status = (_calls or _mx()).quantize(X, fmt, codes, scales, values, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_mx_quantize")


def dq_mx_dequantize(codes, scales, fmt: int, Y, stream=None):
    """Y ([rows, k]) = the values that codes and scales stand for."""
    status = (_calls or _mx()).dequantize(codes, scales, fmt, Y, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_mx_dequantize")


def dq_rmsnorm_quantize(X, gamma, eps: float, fmt: int, codes, scales, residual=None, sum_out=None, values=None, stream=None):
    """h = X + residual; codes and scales of h / sqrt(mean(h^2) + eps) * gamma.  gamma: [k] of X's type or float32, or None.
    sum_out (may be X or residual) receives h, values the quantised output's values; all [rows, k] of X's type."""
    status = (_calls or _mx()).rmsnorm_quantize(X, gamma, eps, fmt, codes, scales, residual, sum_out, values, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_rmsnorm_quantize")


def dq_mx_matmul(a_codes, a_scales, a_fmt: int, w_codes, w_scales, k: int, Y, stream=None):
    """Y ([m, n]) = A W^T for m rows of activations (DQ_MXFP4 or DQ_MXFP8) and n rows of DQ_MXFP4 weights, k values each."""
    status = (_calls or _mx()).matmul(a_codes, a_scales, a_fmt, w_codes, w_scales, k, Y, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_mx_matmul")


def dq_mx_linear(X, a_fmt: int, w_codes, w_scales, Y, workspace, stream=None):
    """Y ([m, n]) = quantised(X) W^T for activations X ([m, k]) and n rows of DQ_MXFP4 weights.  workspace: a buffer of
    dq_mx_linear_workspace(a_fmt, m, k) bytes."""
    status = (_calls or _mx()).linear(X, a_fmt, w_codes, w_scales, Y, workspace, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_mx_linear")


def dq_mx_status(stream=None) -> int:
    """Synchronises the stream; the microscaled operators' status on the current device, which is cleared."""
    return int(load_library().dq_mx_status(_stream_ptr(stream)))


def dq_mx_selftest_bounded_wait(a_codes, a_scales, a_fmt: int, w_codes, w_scales, k: int, Y, step: int, limit_ns: int, stream=None):
    """A product that gives up waiting at a pipeline step: dq_mx_status says DQ_ERR_TIMEOUT afterwards, Y is not valid.  Runs
    the ordinary product first, which checks the arguments."""
    dq_mx_matmul(a_codes, a_scales, a_fmt, w_codes, w_scales, k, Y, stream)
    import torch
    dtype = {torch.float32: DQ_FP32, torch.bfloat16: DQ_BF16, torch.float16: DQ_FP16}[Y.dtype]
    _check(load_library().dq_mx_selftest_bounded_wait(
        a_fmt, a_codes.data_ptr(), a_scales.data_ptr(), Y.shape[0], w_codes.data_ptr(), w_scales.data_ptr(), Y.shape[1], k,
        Y.data_ptr(), dtype, Y.stride(0), step, limit_ns, _stream_ptr(stream)), "dq_mx_selftest_bounded_wait")


# ---------------------------------------------------------------------------
# Attention over a key/value cache in 4 bits (include/dartquant.h says what the calls compute).  Tensors of heads are
# [tokens, heads, head_dim] with contiguous values and any other strides; indices are int32, sums and weights float32.
# ---------------------------------------------------------------------------
def dq_kv_page_bytes(page_size: int, head_dim: int) -> int:
    return int(load_library().dq_kv_page_bytes(page_size, head_dim))


def dq_kv_attention_workspace(head_dim: int) -> int:
    return int(load_library().dq_kv_attention_workspace(head_dim))


def dq_kv_evict_workspace(n_seqs: int, heads: int, keep: int) -> int:
    return int(load_library().dq_kv_evict_workspace(n_seqs, heads, keep))


def dq_kv_pages(n_pages: int, heads: int, head_dim: int, page_size: int, device="cuda"):
    """Memory of n_pages pages of page_size tokens (a power of two from 16 on): uint8 [n_pages, heads, bytes]."""
    import torch
    size = dq_kv_page_bytes(page_size, head_dim)
    if size < 0:
        raise ValueError("pages of %r tokens of %r values: a power of two from 16 to 4096 and 64, 128 or 256 are needed"
                         % (page_size, head_dim))
    return torch.empty((n_pages, heads, size), dtype=torch.uint8, device=device)


class dq_kv_cache:
    """A cache: pages (dq_kv_pages), table (int32 [n_seqs, pages of a sequence]: which page holds its tokens, -1: none) and
    lengths (int32 [n_seqs], a call's own tokens counted).  Holds the tensors, whose contents may change between calls; another
    table or other lengths are another handle."""

    __slots__ = ("pages", "table", "lengths", "head_dim", "page_size", "heads", "n_seqs", "slots", "_struct", "_call")

    def __init__(self, pages, table, lengths, head_dim: int):
        import torch
        if pages.dtype != torch.uint8 or pages.dim() != 3 or not pages.is_contiguous() or not pages.is_cuda:
            raise ValueError("pages: a contiguous CUDA tensor [n_pages, heads, bytes] of uint8 is needed")
        if table.dtype != torch.int32 or table.dim() != 2 or not table.is_contiguous() or table.device != pages.device:
            raise ValueError("table: a contiguous int32 tensor [n_seqs, pages of a sequence] on the pages' device is needed")
        if lengths.dtype != torch.int32 or lengths.shape != table.shape[:1] or not lengths.is_contiguous() or lengths.device != pages.device:
            raise ValueError("lengths: a contiguous int32 tensor [n_seqs] on the pages' device is needed")
        page_size = pages.shape[2] // (head_dim + 8) if head_dim > 0 else 0
        if dq_kv_page_bytes(page_size, head_dim) != pages.shape[2]:
            raise ValueError("pages: %d bytes are no page of heads of %r values" % (pages.shape[2], head_dim))
        if pages.shape[1] < 1 or table.shape[1] < 1:
            raise ValueError("a cache has at least one head, and a table at least one column")
        struct = dq_kv_cache_t(pages.data_ptr(), pages.shape[0], table.data_ptr(), lengths.data_ptr(), table.shape[0],
                               table.shape[1], pages.shape[1], head_dim, page_size)
        for name, value in (("pages", pages), ("table", table), ("lengths", lengths), ("head_dim", head_dim), ("page_size", page_size),
                            ("heads", pages.shape[1]), ("n_seqs", table.shape[0]), ("slots", table.shape[1] * page_size),
                            ("_struct", struct), ("_call", (C.addressof(struct), pages.get_device()))):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):
        raise AttributeError("%s of a cache is fixed: make another handle" % name)


def dq_qk_norm_rope(Q, K, positions, inv_freq, Q_out, K_out, q_gamma=None, k_gamma=None, eps: float = 1e-6, flags: int = DQ_QK_NORM,
                    stream=None):
    """Queries and keys of each head: norm (DQ_QK_NORM), rotation by position, Hadamard rotation (DQ_QK_HADAMARD).  positions:
    [tokens]; inv_freq: [rotated values / 2], or None; gamma: [head_dim] of Q's type or float32; K and K_out may be None, outputs
    their inputs."""
    status = (_calls or _mx()).qk_norm_rope(Q, K, positions, inv_freq, Q_out, K_out, q_gamma, k_gamma, eps, flags, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_qk_norm_rope")


def dq_kv_append(K, V, cache, starts=None, k_values=None, v_values=None, positions=None, slot_positions=None, stream=None):
    """Quantises K and V into the cache, as each sequence's last tokens: rows starts[b] to starts[b + 1], or equally many each.
    k_values, v_values (may be K and V): what the codes stand for.  slot_positions ([n_seqs, heads, cache.slots]) receives
    positions ([tokens]; None: the slots' numbers)."""
    status = (_calls or _mx()).append(K, V, cache, starts, k_values, v_values, positions, slot_positions, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_kv_append")


def dq_kv_dequantize(cache, K, V, starts=None, stream=None):
    """K and V = what the cache holds for each sequence's last tokens."""
    status = (_calls or _mx()).kv_dequantize(cache, K, V, starts, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_kv_dequantize")


def dq_kv_attention(Q, cache, scale: float, out, workspace, starts=None, lse=None, stream=None):
    """out = softmax(scale q k^T) v of each sequence's last tokens over its cache.  workspace: dq_kv_attention_workspace(head_dim)
    bytes, zeros before their first use.  lse ([tokens, Q's heads]): the logarithms of the sums."""
    status = (_calls or _mx()).attention(Q, cache, scale, out, workspace, starts, lse, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_kv_attention")


def dq_kv_attention_weights(Q, lse, cache, scale: float, weights_out, weights=None, starts=None, stream=None):
    """weights_out ([n_seqs, heads, cache.slots]) = weights (None: zeros; new slots start at zero) + the probability that each
    slot received from these queries.  weights_out may be weights."""
    status = (_calls or _mx()).attention_weights(Q, lse, cache, scale, weights_out, weights, starts, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_kv_attention_weights")


def dq_kv_evict(cache, weights, positions, keep: int, recent: int, weights_out, positions_out, lengths_out, workspace, stream=None):
    """Leaves each head of a sequence its `recent` last positions and the slots with the largest weights, `keep` in all, in the slots
    below `keep`.  The outputs may be the inputs (lengths_out: cache.lengths).  workspace: dq_kv_evict_workspace(...) bytes."""
    status = (_calls or _mx()).evict(cache, weights, positions, keep, recent, weights_out, positions_out, lengths_out, workspace, stream)
    if status != DQ_OK:
        raise DartQuantError(status, "dq_kv_evict")


def dq_version() -> str:
    return load_library().dq_version().decode()
