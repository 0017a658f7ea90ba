"""MI355X (gfx950) skew-symmetric LTL^T factorization and Pfaffian.

Thin Python binding over the C ABI of ``libltlt.so`` (``include/ltlt.h``):
it only checks layouts and marshals pointers, sizes and the current HIP
stream; every step of the computation runs in the library's gfx950 kernels.
PyTorch supplies device memory and streams.

Matrices are column-major (the Fortran convention): pass a 2-D tensor ``A``
with ``A.stride(0) == 1`` and ``A.stride(1) == lda >= n`` (for example
``torch.empty_strided((n, n), (1, lda), ...)`` or ``X.t().contiguous().t()``),
so that ``A[i, j]`` is element (i, j).  A row-major tensor is rejected: read as
column-major it would be X^T = -X (same L and P, T negated, Pf times
(-1)^(n/2)).

If the library is not built, or no GPU is visible, every call raises; there
is no CPU fallback.

Calls are asynchronous.  ``factor``, ``pfaffian_direct`` and ``solve`` run
device-side waits that are bounded; when one gives up, the results of that
call are poisoned (NaN factor columns, log|Pf| NaN with sign 0) and a sticky
per-device flag is raised.  Pass ``check=True`` to synchronize and raise
``LtltError`` at once, or call ``device_status()`` later: it raises if any
call since the previous ``device_status()`` failed.
"""
from __future__ import annotations

import array
import ctypes
import functools
import operator
import os
import threading

__all__ = [
    "LIB_PATH",
    "load",
    "factor",
    "pfaffian",
    "factor_batched",
    "skew_update",
    "device_status",
    "test_force_timeout",
    "profile_enable",
    "profile_read",
    "release_workspace",
    "conv_out_size",
    "convgemm",
    "linear",
    "linear_backward",
    "linear_choice",
    "grad_norm",
    "clip_grad_norm",
    "LtltError",
    "F64",
    "F32",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libltlt.so")
F64, F32, C128, C64 = 0, 1, 2, 3
BATCHED_MAX_N = 64
_lock = threading.Lock()
_lib = None

_SYMBOLS = {
    "ltlt_factor": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                     ctypes.c_void_p], ctypes.c_int),
    "ltlt_factor_nb": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                        ctypes.c_int, ctypes.c_void_p], ctypes.c_int),
    "ltlt_pfaffian": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int),
    "ltlt_pfaffian_complex": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int),
    "ltlt_factor_batched": ([ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                             ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                             ctypes.c_void_p], ctypes.c_int),
    "ltlt_skew_update": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                          ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int,
                          ctypes.c_void_p], ctypes.c_int),
    "ltlt_device_status": ([ctypes.c_void_p], ctypes.c_int),
    "ltlt_profile_enable": ([ctypes.c_int], ctypes.c_int),
    "ltlt_profile_read": ([ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int),
    "ltlt_release_workspace": ([], ctypes.c_int),
    "ltlt_set_cooperative_panels": ([ctypes.c_int], ctypes.c_int),
    "ltlt_mfma_probe": ([ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int),
    "ltlt_pfaffian_direct": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                              ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int),
    "ltlt_test_force_timeout": ([ctypes.c_int], ctypes.c_int),
    "ltlt_factor_noalloc": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                             ctypes.c_void_p], ctypes.c_int),
    "ltlt_solve": ([ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_int64,
                    ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p], ctypes.c_int),
    # include/convgemm.h
    "convgemm_out_size": ([ctypes.c_int] * 4, ctypes.c_int),
    "convgemm_choice": ([ctypes.c_int] * 9 + [ctypes.c_void_p], ctypes.c_int),
    "convgemm_f32": ([ctypes.c_int] * 9 + [ctypes.c_void_p] * 3 + [ctypes.c_int] * 4 + [ctypes.c_void_p],
                     ctypes.c_int),
    # include/linear.h
    "convgemm_linear_workspace": ([ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_int] * 2, ctypes.c_int64),
    "convgemm_linear_choice": ([ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.c_void_p], ctypes.c_int),
    "convgemm_linear": ([ctypes.c_int] + [ctypes.c_int64] * 3
                        + [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                           ctypes.c_void_p, ctypes.c_int] + [ctypes.c_void_p, ctypes.c_int64] * 4
                        + [ctypes.c_void_p], ctypes.c_int),
    "convgemm_linear_backward_workspace": ([ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_int] * 3, ctypes.c_int64),
    "convgemm_linear_backward": ([ctypes.c_int] + [ctypes.c_int64] * 3
                                 + [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64]
                                 + [ctypes.c_void_p, ctypes.c_int64] * 3 + [ctypes.c_int]
                                 + [ctypes.c_void_p, ctypes.c_int64] * 2
                                 + [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p], ctypes.c_int),
    "convgemm_grad_workspace": ([ctypes.c_int], ctypes.c_int64),
    "convgemm_grad_norm": ([ctypes.c_int] + [ctypes.c_void_p] * 5 + [ctypes.c_int64, ctypes.c_void_p], ctypes.c_int),
    "convgemm_grad_clip": ([ctypes.c_int] + [ctypes.c_void_p] * 4 + [ctypes.c_double] + [ctypes.c_void_p] * 2
                           + [ctypes.c_int64, ctypes.c_void_p], ctypes.c_int),
}


class LtltError(RuntimeError):
    """A nonzero return code of the C ABI."""

    def __init__(self, fn: str, code: int):
        self.code = code
        if code <= -3000 and code > -4000:
            what = "a device-side bounded wait gave up"
        elif code == -2000:
            what = "size not supported on this device"
        elif code == -4000:
            what = "X is singular (odd order)"
        elif code == -5000:
            what = "the order needs more than the fixed allocation-free workspace"
        elif code <= -1000:
            what = f"HIP runtime error {-1000 - code}"
        else:
            what = f"argument {-code} is invalid"
        super().__init__(f"{fn} returned {code}: {what}")


def load():
    """Load ``libltlt.so`` (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(
                    f"{LIB_PATH} is missing: build it with `python -m paper_2005_06410_amd.build` "
                    "(the GPU path has no fallback)")
            lib = ctypes.CDLL(LIB_PATH)
            for name, (args, res) in _SYMBOLS.items():
                fn = getattr(lib, name)
                fn.argtypes = args
                fn.restype = res
            _lib = lib
    return _lib


def _check(fn: str, code: int):
    if code != 0:
        raise LtltError(fn, code)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.float64:
        return F64
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.complex128:
        return C128
    if t.dtype == torch.complex64:
        return C64
    raise TypeError("only float64, float32, complex128 and complex64 are supported")


def _stream_ptr(device) -> int:
    torch = _torch()
    return torch.cuda.current_stream(device).cuda_stream


def _require_gpu(t):
    if not t.is_cuda:
        raise ValueError("tensor must live on a GPU (the library has no CPU path)")


def _same_device(A, *others):
    """Every tensor argument must live on A's GPU: a host or other-device
    pointer handed to a kernel faults the device instead of raising."""
    for t in others:
        if t is not None and (not t.is_cuda or t.device != A.device):
            raise ValueError("all tensor arguments must be on the same GPU as A")


def _check_ipiv(ipiv, n: int):
    torch = _torch()
    if ipiv.dtype != torch.int32 or not ipiv.is_contiguous() or ipiv.numel() < n:
        raise ValueError("ipiv must be a contiguous int32 tensor with at least n entries")


def _colmajor_lda(A) -> int:
    if A.dim() != 2 or A.shape[0] != A.shape[1]:
        raise ValueError("A must be a square 2-D tensor")
    n = A.shape[0]
    if n <= 1:
        return max(1, A.stride(1) if A.dim() == 2 else 1)
    if A.stride(0) != 1 or A.stride(1) < n:
        raise ValueError("A must be column-major: stride(0) == 1 and stride(1) = lda >= n "
                         "(a row-major skew matrix would be read as its negation)")
    return A.stride(1)


def factor(A, ipiv=None, nb: int | None = None, check: bool = False):
    """In-place P X P^T = L T L^T of the column-major skew matrix ``A``
    (float64, float32, or complex128 / complex64 for a complex X with
    X^T = -X).

    Returns the int32 pivot tensor (0-based, LAPACK laswp order).  On return
    A's strict lower triangle holds alpha_k at (k+1, k) and L(r, k+1) at (r, k);
    its strict upper triangle is never touched.  ``check=True`` synchronizes
    and raises if a device-side wait gave up (see the module docstring)."""
    torch = _torch()
    _require_gpu(A)
    lda = _colmajor_lda(A)
    n = A.shape[0]
    if ipiv is None:
        ipiv = torch.empty(max(n, 1), dtype=torch.int32, device=A.device)
    _same_device(A, ipiv)
    _check_ipiv(ipiv, n)
    lib = load()
    s = _stream_ptr(A.device)
    if nb is None:
        code = lib.ltlt_factor(n, A.data_ptr(), lda, _dtype_code(A), ipiv.data_ptr(), s)
    else:
        code = lib.ltlt_factor_nb(n, A.data_ptr(), lda, _dtype_code(A), ipiv.data_ptr(), int(nb), s)
    _check("ltlt_factor", code)
    if check:
        device_status(A.device)
    return ipiv[:n] if ipiv.numel() != n else ipiv


def pfaffian(A, ipiv):
    """(logabs, sign) device tensors of Pf(X) from ``factor``'s output; for a
    complex A, (logabs, phase) with phase = Pf/|Pf| a complex128 tensor."""
    torch = _torch()
    _require_gpu(A)
    lda = _colmajor_lda(A)
    n = A.shape[0]
    _same_device(A, ipiv)
    _check_ipiv(ipiv, n)
    logabs = torch.empty(1, dtype=torch.float64, device=A.device)
    lib = load()
    if A.is_complex():
        phase = torch.empty((1, 2), dtype=torch.float64, device=A.device)
        code = lib.ltlt_pfaffian_complex(n, A.data_ptr(), lda, _dtype_code(A), ipiv.data_ptr(), logabs.data_ptr(),
                                         phase.data_ptr(), _stream_ptr(A.device))
        _check("ltlt_pfaffian_complex", code)
        return logabs, torch.view_as_complex(phase)
    sign = torch.empty(1, dtype=torch.int32, device=A.device)
    code = lib.ltlt_pfaffian(n, A.data_ptr(), lda, _dtype_code(A), ipiv.data_ptr(), logabs.data_ptr(),
                             sign.data_ptr(), _stream_ptr(A.device))
    _check("ltlt_pfaffian", code)
    return logabs, sign


def pfaffian_direct(A, nb: int = 0, ipiv=None, check: bool = False):
    """Pf(X) of the column-major skew matrix ``A`` from the even column steps
    only (see ``ltlt_pfaffian_direct``); ``A`` is used as workspace.

    Returns (ipiv int32 (n,), logabs f64 (1,), sign int32 (1,)) device tensors.
    ``check=True`` synchronizes and raises if a device-side wait gave up."""
    torch = _torch()
    _require_gpu(A)
    lda = _colmajor_lda(A)
    n = A.shape[0]
    if ipiv is None:
        ipiv = torch.empty(max(n, 1), dtype=torch.int32, device=A.device)
    _same_device(A, ipiv)
    _check_ipiv(ipiv, n)
    logabs = torch.empty(1, dtype=torch.float64, device=A.device)
    sign = torch.empty(1, dtype=torch.int32, device=A.device)
    code = load().ltlt_pfaffian_direct(n, A.data_ptr(), lda, _dtype_code(A), ipiv.data_ptr(), int(nb),
                                       logabs.data_ptr(), sign.data_ptr(), _stream_ptr(A.device))
    _check("ltlt_pfaffian_direct", code)
    if check:
        device_status(A.device)
    return ipiv[:n], logabs, sign


def solve(A, ipiv, B, check: bool = False):
    """Overwrite B (column-major n or n x nrhs, same dtype and device as A)
    with X^{-1} B from ``factor``'s output (see ``ltlt_solve``).
    ``check=True`` synchronizes and raises if a device-side wait gave up."""
    _require_gpu(A)
    _require_gpu(B)
    lda = _colmajor_lda(A)
    n = A.shape[0]
    _same_device(A, B, ipiv)
    _check_ipiv(ipiv, n)
    if B.dtype != A.dtype:
        raise ValueError("B must have A's dtype")
    if B.dim() == 1:
        nrhs, ldb = 1, max(B.shape[0], 1)
        if B.stride(0) != 1:
            raise ValueError("B must be contiguous")
    elif B.dim() == 2:
        nrhs = B.shape[1]
        if B.shape[0] > 1 and B.stride(0) != 1:
            raise ValueError("B must be column-major")
        ldb = B.stride(1) if nrhs > 1 else max(B.shape[0], 1)
    else:
        raise ValueError("B must be 1-D or 2-D")
    if B.shape[0] != n:
        raise ValueError("B must have n rows")
    code = load().ltlt_solve(n, A.data_ptr(), lda, _dtype_code(A), ipiv.data_ptr(), nrhs, B.data_ptr(), ldb,
                             _stream_ptr(A.device))
    _check("ltlt_solve", code)
    if check:
        device_status(A.device)
    return B


def factor_batched(A, ipiv=None):
    """Factor and take the Pfaffian of every matrix of a (batch, n, n) tensor
    whose matrices are column-major (``A.stride(1) == 1``, ``A.stride(2) == lda``).

    Returns (ipiv (batch, n) int32, logabs (batch,) f64, sign (batch,) int32)."""
    torch = _torch()
    _require_gpu(A)
    if A.dim() != 3 or A.shape[1] != A.shape[2]:
        raise ValueError("A must be (batch, n, n)")
    batch, n = A.shape[0], A.shape[1]
    if n > 1 and (A.stride(1) != 1 or A.stride(2) < n):
        raise ValueError("each matrix must be column-major: stride(1) == 1, stride(2) = lda >= n")
    lda = A.stride(2) if n > 1 else max(1, n)
    strideA = A.stride(0) if batch > 1 else lda * max(n, 1)
    if ipiv is None:
        ipiv = torch.empty((batch, max(n, 1)), dtype=torch.int32, device=A.device)
    _same_device(A, ipiv)
    if (ipiv.dtype != torch.int32 or ipiv.dim() != 2 or ipiv.shape[0] != batch or ipiv.shape[1] < n
            or (n > 1 and ipiv.stride(1) != 1)):
        raise ValueError("ipiv must be an int32 (batch, >= n) tensor with unit stride along each row")
    logabs = torch.empty(batch, dtype=torch.float64, device=A.device)
    sign = torch.empty(batch, dtype=torch.int32, device=A.device)
    lib = load()
    code = lib.ltlt_factor_batched(n, batch, A.data_ptr(), lda, strideA, _dtype_code(A), ipiv.data_ptr(),
                                   ipiv.stride(0), logabs.data_ptr(), sign.data_ptr(), _stream_ptr(A.device))
    _check("ltlt_factor_batched", code)
    return ipiv[:, :n], logabs, sign


def skew_update(C, Lx, Bt, perm=None, offset: int = 0):
    """The trailing-block update on its own (see ``ltlt_skew_update``).

    ``C`` is a column-major tensor view; the m x m block starting ``offset``
    rows and columns into it is updated; ``perm`` (int32, length m) holds
    source indices relative to that block start."""
    torch = _torch()
    _require_gpu(C)
    if C.dim() != 2 or C.stride(0) != 1:
        raise ValueError("C must be column-major")
    m, K = Lx.shape
    ldc = C.stride(1)
    _same_device(C, Lx, Bt, perm)
    for t in (Lx, Bt):
        if t.dim() != 2 or (t.shape[0] > 1 and t.stride(0) != 1):
            raise ValueError("Lx and Bt must be column-major")
        if t.dtype != C.dtype:
            raise ValueError("Lx and Bt must have C's dtype")
    if tuple(Bt.shape) != (m, K):
        raise ValueError("Bt must have Lx's shape (m, K)")
    if offset < 0 or offset + m > min(C.shape[0], C.shape[1]):
        raise ValueError("the m x m block at `offset` must lie inside C")
    if perm is not None and (perm.dtype != torch.int32 or not perm.is_contiguous() or perm.numel() < m):
        raise ValueError("perm must be a contiguous int32 tensor with at least m entries")
    elem = C.element_size()
    ptr = C.data_ptr() + (offset + offset * ldc) * elem
    pp = 0 if perm is None else perm.data_ptr()

    def ld(t):  # leading dimension; a single column may carry any stride
        return max(t.stride(1), 1) if t.shape[1] > 1 else max(t.shape[0], 1)

    lib = load()
    code = lib.ltlt_skew_update(m, ptr, ldc, pp, K, Lx.data_ptr(), ld(Lx), Bt.data_ptr(), ld(Bt),
                                _dtype_code(C), _stream_ptr(C.device))
    _check("ltlt_skew_update", code)


def conv_out_size(h: int, k: int, stride: int = 1, pad: int = 0) -> int:
    """floor((h - k + 2 pad)/stride) + 1 (``convgemm_out_size``); raises when
    the window does not fit the padded input."""
    r = load().convgemm_out_size(int(h), int(k), int(stride), int(pad))
    if r < 1:
        raise ValueError(f"no output for h={h} k={k} stride={stride} pad={pad}")
    return r


def conv_choice(kn: int, kh: int, kw: int, ci: int, hi: int, wi: int, b: int, stride: int = 1, pad: int = 0):
    """The kernel that ``convgemm`` takes by itself for a layer, as (family,
    mt, nt, share): see ``convgemm_choice``.  Host only."""
    out = (ctypes.c_int * 4)()
    code = load().convgemm_choice(*(int(v) for v in (kn, kh, kw, ci, hi, wi, b, stride, pad)), ctypes.addressof(out))
    _check("convgemm_choice", code)
    return tuple(out)


def _leftmost_fastest(t, name):
    """The convolution tensors are stored with the leftmost index fastest."""
    torch = _torch()
    if t.dtype != torch.float32 or t.dim() != 4:
        raise TypeError(f"{name} must be a 4-d float32 tensor")
    if not t.permute(3, 2, 1, 0).is_contiguous():
        raise ValueError(f"{name} must be stored leftmost index fastest (strides (1, d0, d0 d1, d0 d1 d2))")


def convgemm(F, I, stride: int = 1, pad: int = 0, out=None, accumulate: bool = False, path: int = 0,
             tile=(0, 0)):
    """O = conv(F, I) (or O += conv(F, I) with ``accumulate``) by the
    implicit-im2col GEMM of ``convgemm_f32``.

    F: (kn, kh, kw, ci) and I: (hi, wi, ci, b) float32 GPU tensors stored with
    the leftmost index fastest (a numpy Fortran-order array's layout).
    Returns O (kn, ho, wo, b) in the same storage (``out`` if given).
    ``path`` (1 LDS-staged, 2 register-direct) and ``tile`` = (mt, nt) force a
    kernel and workgroup tile (tests and tuning); 0 / (0, 0) choose them."""
    torch = _torch()
    _require_gpu(I)
    _same_device(I, F, out)
    _leftmost_fastest(F, "F")
    _leftmost_fastest(I, "I")
    kn, kh, kw, ci = F.shape
    hi, wi, ci2, b = I.shape
    if ci2 != ci:
        raise ValueError("F and I disagree on the channel count")
    ho, wo = conv_out_size(hi, kh, stride, pad), conv_out_size(wi, kw, stride, pad)
    if out is None:
        flat = torch.empty(max(kn * ho * wo * b, 1), dtype=torch.float32, device=I.device)
        out = flat[:kn * ho * wo * b].as_strided((kn, ho, wo, b), (1, kn, kn * ho, kn * ho * wo))
    else:
        _leftmost_fastest(out, "out")
        if tuple(out.shape) != (kn, ho, wo, b):
            raise ValueError(f"out must have shape {(kn, ho, wo, b)}")
    mt, nt = tile
    code = load().convgemm_f32(kn, kh, kw, ci, hi, wi, b, int(stride), int(pad), F.data_ptr(), I.data_ptr(),
                               out.data_ptr(), int(bool(accumulate)), int(path), int(mt), int(nt),
                               _stream_ptr(I.device))
    _check("convgemm_f32", code)
    return out


# Layer operators (include/linear.h).  A call of a few tokens is bound by what
# happens on the host, so these bindings ask each tensor each thing once.
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
_layer_codes = {}


def _layer_dtype(dtype) -> int:
    code = _layer_codes.get(dtype)
    if code is None:
        torch = _torch()
        _layer_codes.update({torch.float32: 1, torch.bfloat16: 4, torch.float16: 5})
        code = _layer_codes.get(dtype)
        if code is None:
            raise TypeError("only float32, bfloat16 and float16 are supported")
    return code


def _activation(name) -> int:
    code = ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    return code


def _layer_input(X):
    """(ci, t, leading dimension, dtype, its code, GPU index) of a layer's input."""
    _require_gpu(X)
    if X.dim() != 2:
        raise ValueError("X must be (ci, t)")
    ci, t = X.shape
    dtype, dev = X.dtype, X.get_device()
    return ci, t, _columns(X, ci, t, "X", dtype, dev), dtype, _layer_dtype(dtype), dev


def _columns(v, rows: int, cols: int, name: str, dtype, dev: int) -> int:
    """The leading dimension of a (rows, cols) tensor stored with its first
    index fastest, of the given dtype on the given GPU."""
    if v.shape != (rows, cols):
        raise ValueError(f"{name} must have shape {(rows, cols)}")
    if v.dtype != dtype:
        raise TypeError(f"{name} must have X's dtype")
    if v.get_device() != dev:
        raise ValueError("all tensor arguments must be on the same GPU")
    s0, s1 = v.stride()
    if (rows > 1 and s0 != 1) or (cols > 1 and s1 < max(rows, 1)):
        raise ValueError(f"{name} must be stored leftmost index fastest: stride(0) == 1, stride(1) >= {rows}")
    return s1 if cols > 1 else max(rows, 1)


def _meet(a: int, alen: int, alines: int, ald: int, b: int, blen: int, blines: int, bld: int) -> bool:
    """Whether two sets of lines share a value: lines of `len` values, `ld` apart,
    from the addresses a and b (in values).  Lines at different distances, both with
    gaps, are taken for disjoint."""
    if alen * alines == 0 or blen * blines == 0:
        return False
    if a + (alines - 1) * ald + alen <= b or b + (blines - 1) * bld + blen <= a:
        return False
    if alines == 1 or ald == alen:                   # a has no gaps: one line
        alen, alines = (alines - 1) * ald + alen, 1
    if blines == 1 or bld == blen:
        blen, blines = (blines - 1) * bld + blen, 1
    if blines == 1:
        a, alen, alines, ald, b, blen, blines, bld = b, blen, blines, bld, a, alen, alines, ald
    if alines == 1:                                  # the first line of b that ends behind a's start
        k = 0 if b + blen > a else (a - b - blen) // bld + 1
        return k < blines and b + k * bld < a + alen
    if ald != bld:
        return False
    d = (b - a) % ald                                # within the same period
    return d < alen or d + blen > ald


def _weights(F, ci: int, dtype, dev: int):
    """(kn, order, leading dimension) of weights with either index fastest."""
    if F.dim() != 2:
        raise ValueError("F must be (kn, ci)")
    if F.dtype != dtype:
        raise TypeError("F must have X's dtype")
    if F.get_device() != dev:
        raise ValueError("all tensor arguments must be on the same GPU")
    kn, fci = F.shape
    if fci != ci:
        raise ValueError("F and X disagree on the number of inputs")
    s0, s1 = F.stride()
    if (ci <= 1 or s1 == 1) and (kn <= 1 or s0 >= max(ci, 1)):
        return kn, 1, s0 if kn > 1 else max(ci, 1)
    if (kn <= 1 or s0 == 1) and (ci <= 1 or s1 >= max(kn, 1)):
        return kn, 0, s1 if ci > 1 else max(kn, 1)
    raise ValueError("F must have one index with stride 1 and no overlap along the other")


def _aligned(code: int, lds: int, ptrs: int) -> int:
    """Whether leading dimensions (or-ed together) and addresses (likewise) are
    whole 16 bytes, and the former below the direct loads' limit."""
    size = 4 if code == 1 else 2
    return int(not (lds * size | ptrs) & 15 and lds < 1 << 20)


def _raw_stream(dev: int) -> int:
    """The current stream of GPU `dev`, by torch's direct query where it has one."""
    c = _torch()._C
    raw = getattr(c, "_cuda_getCurrentRawStream", None)
    return raw(dev) if raw is not None else _stream_ptr(dev)


@functools.lru_cache(maxsize=4096)
def _scratch_bytes(fn: str, dev: int, *sizes) -> int:
    """What the library answers for these sizes on GPU `dev`."""
    with _torch().cuda.device(dev):
        need = getattr(load(), fn)(*sizes)
    if need < 0:
        raise ValueError(f"sizes out of range (argument {-need} of {fn})")
    return need


def _scratch(need: int, like):
    """Workspace of a call, from torch's allocator: stream-ordered like the call."""
    return like.new_empty(need, dtype=_torch().uint8)


def _launch(fn: str, dev: int, *args):
    """Calls the library with the current stream, on the tensors' GPU."""
    torch = _torch()
    f = getattr(load(), fn)
    if torch.cuda.current_device() == dev:
        _check(fn, f(*args, _raw_stream(dev)))
    else:
        with torch.cuda.device(dev):
            _check(fn, f(*args, _raw_stream(dev)))


def linear(F, X, bias=None, activation: str = "none", residual=None, out=None, keep_pre: bool = False):
    """O = act(F X + bias) + residual, one matrix product with the rest in its
    epilogue (``convgemm_linear``).

    F: (kn, ci), either index fastest (the convolution's filters, or a row-major
    weight as it is); X: (ci, t) and ``residual`` (kn, t) stored with the
    leftmost index fastest (the transposed view of row-major activations);
    ``bias``: (kn,).  All float32, bfloat16 or float16; sums and epilogue are
    fp32, and each result is rounded once.  ``activation``: none, relu, gelu,
    gelu_tanh or silu.

    Returns O (kn, t) in the same storage (``out`` if given; it may be
    ``residual`` itself and overlap no other input), or (O, Z) with the pre-activation
    Z = F X + bias for ``linear_backward`` where ``keep_pre`` is set.  Nothing is
    recorded for torch's automatic differentiation, whatever the tensors require:
    gradients come from ``linear_backward``."""
    ci, t, ldx, dtype, code, dev = _layer_input(X)
    kn, order, ldf = _weights(F, ci, dtype, dev)
    act = _activation(activation)
    bp = rp = zp = 0
    ldr = 1
    if bias is not None:
        if bias.shape != (kn,) or (kn > 1 and bias.stride(0) != 1):
            raise ValueError(f"bias must be a contiguous tensor of {kn} values")
        if bias.dtype != dtype:
            raise TypeError("bias must have X's dtype")
        if bias.get_device() != dev:
            raise ValueError("all tensor arguments must be on the same GPU")
        bp = bias.data_ptr()
    if residual is not None:
        ldr = _columns(residual, kn, t, "residual", dtype, dev)
        rp = residual.data_ptr()
    if out is None:
        out = X.new_empty_strided((kn, t), (1, max(kn, 1)))
        ldo = max(kn, 1)
    else:
        ldo = _columns(out, kn, t, "out", dtype, dev)
        size, op = out.element_size(), out.data_ptr()
        inputs = [(X.data_ptr(), ci, t, ldx), (F.data_ptr(), *((ci, kn) if order else (kn, ci)), ldf), (bp, kn if bp else 0, 1, 1),
                  (rp, kn if rp and not (rp == op and ldr == ldo) else 0, t, ldr)]
        if any([_meet(op // size, kn, t, ldo, p // size, rows, lines, ld) for p, rows, lines, ld in inputs]):
            raise ValueError("out may not overlap an input other than residual itself")
    if keep_pre:
        Z = X.new_empty_strided((kn, t), (1, max(kn, 1)))
        zp = Z.data_ptr()
    fp, xp = F.data_ptr(), X.data_ptr()
    need = _scratch_bytes("convgemm_linear_workspace", dev, code, kn, ci, t, order,
                          _aligned(code, ldf | ldx, fp | xp))
    ws = _scratch(need, X) if need else None
    _launch("convgemm_linear", dev, code, kn, ci, t, fp, order, ldf, xp, ldx, bp, act, rp, ldr, zp,
            max(kn, 1), out.data_ptr(), ldo, ws.data_ptr() if need else 0, need)
    return (out, Z) if keep_pre else out


def linear_choice(dtype, kn: int, ci: int, t: int, f_order: int = 1, aligned: bool = True):
    """The kernel that ``linear`` takes for a layer, as (family, tile outputs,
    tile tokens, splits, copies, kernel): see ``convgemm_linear_choice``.  Host only;
    ``f_order`` 1 for row-major weights, 0 for the convolution's order."""
    out = (ctypes.c_int * 6)()
    _check("convgemm_linear_choice", load().convgemm_linear_choice(
        _layer_dtype(dtype), int(kn), int(ci), int(t), int(f_order), int(bool(aligned)), ctypes.addressof(out)))
    return tuple(out)


def linear_backward(F, X, dO, pre=None, activation: str = "none", needs=(True, True, True)):
    """(dX, dF, dbias) of ``linear`` from dO = dL/dO (kn, t), stored like O
    (``convgemm_linear_backward``); the residual's gradient is dO itself.

    ``pre`` is the Z that ``linear(..., keep_pre=True)`` returned; without an
    activation it is not needed.  dX is stored like X, dF in F's order.  Between
    the two products dO act'(Z) is rounded to the layer's type once (fp16: times a
    power of two, so that its range does not matter).
    ``needs`` leaves out what is not wanted (None is returned in its place)."""
    ci, t, ldx, dtype, code, dev = _layer_input(X)
    kn, order, ldf = _weights(F, ci, dtype, dev)
    act = _activation(activation)
    lddo = _columns(dO, kn, t, "dO", dtype, dev)
    zp, ldz = 0, 1
    if act:
        if pre is None:
            raise ValueError("an activation's gradient needs the pre-activation (pre)")
        ldz = _columns(pre, kn, t, "pre", dtype, dev)
        zp = pre.data_ptr()
    dX = dF = db = None
    xp = fp = bp = 0
    if needs[0]:
        dX = X.new_empty_strided((ci, t), (1, max(ci, 1)))
        xp = dX.data_ptr()
    if needs[1]:
        dF = X.new_empty_strided((kn, ci), (max(ci, 1), 1) if order else (1, max(kn, 1)))
        fp = dF.data_ptr()
    if needs[2]:
        db = X.new_empty(kn)
        bp = db.data_ptr()
    need = _scratch_bytes("convgemm_linear_backward_workspace", dev, code, kn, ci, t, order, act,
                          _aligned(code, ldf | ldx | lddo, F.data_ptr() | X.data_ptr() | dO.data_ptr()))
    ws = _scratch(need, X) if need else None
    _launch("convgemm_linear_backward", dev, code, kn, ci, t, F.data_ptr(), order, ldf, X.data_ptr(), ldx, dO.data_ptr(),
            lddo, zp, ldz, act, xp, max(ci, 1), fp, max(ci if order else kn, 1), bp, ws.data_ptr() if need else 0, need)
    return dX, dF, db


def _dense(t) -> bool:
    """Whether t's values fill its memory without gaps or overlap, in any order."""
    if t.is_contiguous():
        return True
    want = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != want:
            return False
        want *= size
    return True


def _grad_list(grads, what):
    """(tensors, GPU index, whether all are contiguous, and as host arrays their
    addresses, sizes and types); one C-level pass over the list per question."""
    grads = list(grads)
    if not grads:
        raise ValueError(f"no {what}")
    T = _torch().Tensor
    devs = set(map(T.get_device, grads))
    dev = devs.pop()
    if dev < 0 or devs:
        raise ValueError(f"all {what} must be on the same GPU (the library has no CPU path)")
    plain = all(map(T.is_contiguous, grads))
    if not plain and not all(map(_dense, grads)):
        raise ValueError(f"{what} must be stored without gaps or overlap")
    dtypes = list(map(operator.attrgetter("dtype"), grads))
    if dtypes.count(dtypes[0]) == len(dtypes):
        codes = array.array("i", (_layer_dtype(dtypes[0]),)) * len(grads)
    else:
        codes = array.array("i", map(_layer_dtype, dtypes))
    return grads, dev, plain, array.array("Q", map(T.data_ptr, grads)), array.array("q", map(T.numel, grads)), codes


def grad_norm(grads):
    """The 2-norm of all tensors of ``grads`` together, one float32 value on
    their GPU (``convgemm_grad_norm``); squares are summed in fp64.

    Tensors are float32, bfloat16 or float16 (mixed as they come), of any shape,
    stored without gaps in any order.  An empty list is refused: it names no GPU."""
    return _norm_and_clip(grads, None, None)


def clip_grad_norm(grads, max_norm: float, out=None):
    """Scales ``grads`` by c = min(1, max_norm / norm) with their joint norm
    (``convgemm_grad_clip``), in place or into the tensors ``out`` (the same
    sizes, types and order in memory).  Returns the norm before scaling, as
    ``grad_norm`` does; nothing is copied to the host.

    An infinite gradient makes c zero and a NaN makes it NaN; a norm above fp32's
    range is returned as infinity but scales by its value.  The tensors to be
    scaled may not overlap one another (the same one twice is refused)."""
    if not max_norm >= 0:
        raise ValueError("max_norm must be at least 0")
    return _norm_and_clip(grads, float(max_norm), out)


def _norm_and_clip(grads, max_norm, out):
    grads, dev, plain, ptrs, sizes, codes = _grad_list(grads, "gradients")
    optrs = ptrs
    if out is not None:
        outs, odev, oplain, optrs, osizes, ocodes = _grad_list(out, "outputs")
        if odev != dev or osizes != sizes or ocodes != codes or (not (plain and oplain) and any(
                [o.shape != g.shape or (o.stride() != g.stride() and not (o.is_contiguous() and g.is_contiguous()))
                 for o, g in zip(outs, grads)])):
            raise ValueError("out must have the gradients' sizes, types, order in memory and GPU")
    if max_norm is not None:
        names = set(optrs)
        if len(names) != len(optrs) and len({p for p, n in zip(optrs, sizes) if n}) != len(sizes) - sizes.count(0):
            raise ValueError("a tensor to be scaled is named twice")
        if out is not None and not names.isdisjoint(ptrs):
            where = {p: i for i, (p, n) in enumerate(zip(ptrs, sizes)) if n}
            if any(n and where.get(p, i) != i for i, (p, n) in enumerate(zip(optrs, sizes))):
                raise ValueError("an output is another gradient")
    norm = grads[0].new_empty((), dtype=_torch().float32)
    count = len(grads)
    need = _scratch_bytes("convgemm_grad_workspace", dev, count)
    ws = _scratch(need, grads[0])
    g, o, n, d = [v.buffer_info()[0] for v in (ptrs, optrs, sizes, codes)]
    if max_norm is None:
        _launch("convgemm_grad_norm", dev, count, g, n, d, norm.data_ptr(), ws.data_ptr(), need)
    else:
        _launch("convgemm_grad_clip", dev, count, g, o, n, d, max_norm, norm.data_ptr(), ws.data_ptr(), need)
    return norm


def device_status(device=None):
    """Synchronize and raise if a device-side bounded wait of any call on the
    device gave up since the previous ``device_status`` (clears that flag)."""
    torch = _torch()
    lib = load()
    dev = device if device is not None else torch.cuda.current_device()
    with torch.cuda.device(dev):
        _check("ltlt_device_status", lib.ltlt_device_status(_stream_ptr(dev)))


def test_force_timeout(on: bool = True):
    """Failure-path tests only: while on, every factor / pfaffian_direct /
    solve call behaves as if a device-side wait had given up at its start
    (see ``ltlt_test_force_timeout``)."""
    _check("ltlt_test_force_timeout", load().ltlt_test_force_timeout(1 if on else 0))


def profile_enable(on=True):
    """Record per-launch event timings: True (every launch), "update" (the
    trailing-update launches only), or False (stop)."""
    mode = 2 if on == "update" else (1 if on else 0)
    _check("ltlt_profile_enable", load().ltlt_profile_enable(mode))


def profile_read():
    """{kind: (launches, ms, flops)} for kinds panel, update, commit, other."""
    lib = load()
    launches = (ctypes.c_int64 * 4)()
    ms = (ctypes.c_double * 4)()
    flops = (ctypes.c_double * 4)()
    k = lib.ltlt_profile_read(4, launches, ms, flops)
    if k < 0:
        raise LtltError("ltlt_profile_read", k)
    names = ["panel", "update", "commit", "other"]
    return {names[i]: (int(launches[i]), float(ms[i]), float(flops[i])) for i in range(k)}


def release_workspace():
    _check("ltlt_release_workspace", load().ltlt_release_workspace())


def set_cooperative_panels(on: bool = True):
    """Launch the panel kernels with the runtime's cooperative launch (its
    co-residency guarantee, for devices shared with other work) or, the
    default, as ordinary launches (see ``ltlt_set_cooperative_panels``)."""
    _check("ltlt_set_cooperative_panels", load().ltlt_set_cooperative_panels(1 if on else 0))


def mfma_probe(dtype: str = "f64", iters: int = 20000, device=None) -> float:
    """Sustained TFLOP/s of a register-only MFMA loop on the device (see
    ``ltlt_mfma_probe``)."""
    torch = _torch()
    dev = device if device is not None else torch.cuda.current_device()
    out = ctypes.c_double(0.0)
    code = load().ltlt_mfma_probe(0 if dtype == "f64" else 1, int(iters), ctypes.addressof(out), _stream_ptr(dev))
    _check("ltlt_mfma_probe", code)
    return float(out.value)
