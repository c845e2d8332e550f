"""Python binding of the rank-compensation hot path (liblrc.so, gfx950).

Argument marshalling only: torch tensors are checked for device, dtype and
layout, their data pointers and torch's current stream are passed to the C
ABI declared in include/lrc.h, and every computation runs in the library's
HIP kernels.  There is no CPU fallback: if the library is missing this
module raises on first use.

Precision follows the tensors' dtype: float64 -> FP64, float32 -> FP32,
float16 -> FP16 (FP32 accumulation); the output-head calls also take bfloat16.

Every call returns plain tensors and records nothing for autograd, also for
inputs that require a gradient.  The distillation loss (distill,
distill_backward: by the student's logits), the norm (rms_norm_backward) and
the adapters (adapter_backward) have a gradient; the 4-bit product and the
8-bit norm have no backward call.
"""
from __future__ import annotations

import ctypes
import math
import os
import re

HERE = os.path.dirname(os.path.abspath(__file__))
# LRC_LIBRARY selects another build of the same sources (the host-sanitized build)
LIB_PATH = os.environ.get("LRC_LIBRARY") or os.path.join(HERE, "liblrc.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "lrc.h")

FP64, FP32, FP16, BF16, E4M3 = 0, 1, 2, 3, 4
PATH_AUTO, PATH_STREAM, PATH_MFMA = 0, 1, 2
CERT_MATRIX, CERT_TT = 0, 1
ERRORS = {-1: "EINVAL", -2: "EOVERFLOW", -3: "EHIP", -4: "ENOMEM", -5: "ENODEV", -6: "ENUMERIC"}
PREC_NAMES = {"fp64": FP64, "fp32": FP32, "fp16": FP16}


class LrcError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


_i64 = ctypes.c_int64
_vp = ctypes.c_void_p


class CertArgs(ctypes.Structure):
    _fields_ = [
        ("kind", ctypes.c_int), ("prec", ctypes.c_int),
        ("m", _i64), ("n", _i64), ("k", _i64),
        ("sigma", ctypes.POINTER(ctypes.c_double)), ("n_sigma", _i64),
        ("U", _vp), ("s", _vp), ("V", _vp),
        ("Uh", _vp), ("sh", _vp), ("Vh", _vp),
        ("A", _vp),
        ("d", ctypes.c_int),
        ("dims", ctypes.POINTER(_i64)),
        ("T", _vp),
        ("ranks_base", ctypes.POINTER(_i64)), ("cores_base", ctypes.POINTER(_vp)),
        ("ranks_aug", ctypes.POINTER(_i64)), ("cores_aug", ctypes.POINTER(_vp)),
        ("cores_aug_h", ctypes.POINTER(_vp)),
    ]


class CertResult(ctypes.Structure):
    _fields_ = [
        ("E_base", ctypes.c_double), ("E_aug", ctypes.c_double), ("eta", ctypes.c_double),
        ("err_new", ctypes.c_double), ("gain", ctypes.c_double), ("margin", ctypes.c_double),
        ("norm_ref", ctypes.c_double),
        ("bytes_base", _i64), ("bytes_aug", _i64),
        ("certified", ctypes.c_int), ("acc_nonincrease", ctypes.c_int), ("acc_win", ctypes.c_int),
        ("mem_win", ctypes.c_int), ("practical_win", ctypes.c_int), ("outcome", ctypes.c_int),
    ]


class Quality(ctypes.Structure):
    _fields_ = [("rel_err", ctypes.c_double), ("psnr", ctypes.c_double), ("ssim", ctypes.c_double),
                ("sam", ctypes.c_double), ("sam_pixels", _i64), ("pixels", _i64), ("bands", _i64)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_12969_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    L.lrc_matrix_apply.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, ctypes.c_int]
    L.lrc_matrix_apply.restype = ctypes.c_int
    L.lrc_matrix_apply_noalloc.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, ctypes.c_int]
    L.lrc_matrix_apply_noalloc.restype = ctypes.c_int
    L.lrc_mfma_ceiling.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double)]
    L.lrc_mfma_ceiling.restype = ctypes.c_int
    L.lrc_matrix_apply_path.argtypes = [_i64, _i64, _i64, _i64, ctypes.c_int]
    L.lrc_matrix_apply_path.restype = ctypes.c_int
    L.lrc_set_apply_path.argtypes = [ctypes.c_int]
    L.lrc_set_apply_path.restype = ctypes.c_int
    L.lrc_tt_reconstruct.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                                     ctypes.c_int, _vp, ctypes.c_int]
    L.lrc_tt_reconstruct.restype = ctypes.c_int
    L.lrc_certify.argtypes = [ctypes.POINTER(CertArgs), ctypes.POINTER(CertResult)]
    L.lrc_certify.restype = ctypes.c_int
    L.lrc_round.argtypes = [_vp, _vp, _i64, ctypes.c_int, ctypes.POINTER(_i64)]
    L.lrc_round.restype = ctypes.c_int
    L.lrc_tt_left_orthogonalize.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                                            ctypes.c_int]
    L.lrc_tt_left_orthogonalize.restype = ctypes.c_int
    L.lrc_band_quality.argtypes = [_vp, _vp, _i64, _i64, ctypes.c_int, ctypes.c_double, ctypes.POINTER(Quality)]
    L.lrc_band_quality.restype = ctypes.c_int
    L.lrc_tt_quality.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_i64), ctypes.POINTER(_i64), ctypes.c_int,
                                 ctypes.c_int, _vp, ctypes.c_double, ctypes.POINTER(Quality)]
    L.lrc_tt_quality.restype = ctypes.c_int
    L.lrc_tt_memory_matched_rank.argtypes = [ctypes.POINTER(_i64), ctypes.c_int, _i64, ctypes.POINTER(_i64)]
    L.lrc_tt_memory_matched_rank.restype = _i64
    L.lrc_rsvd.argtypes = [_vp, _i64, _i64, _vp, _i64, ctypes.c_int, _i64, _vp, _vp, _vp]
    L.lrc_rsvd.restype = ctypes.c_int
    L.lrc_tt_rsvd.argtypes = [_vp, ctypes.POINTER(_i64), ctypes.POINTER(_i64), ctypes.c_int, ctypes.POINTER(_vp),
                              ctypes.POINTER(_i64), ctypes.c_int, ctypes.POINTER(_vp), _vp]
    L.lrc_tt_rsvd.restype = ctypes.c_int
    L.lrc_q4_row_bytes.argtypes = [_i64]
    L.lrc_q4_row_bytes.restype = _i64
    L.lrc_q4_storage_bytes.argtypes = [_i64, _i64, _i64, ctypes.c_int]
    L.lrc_q4_storage_bytes.restype = _i64
    L.lrc_q4_quantize.argtypes = [_vp, _i64, _i64, _i64, _i64, ctypes.c_int, _vp, _vp, ctypes.c_int, _vp,
                                  ctypes.POINTER(_i64)]
    L.lrc_q4_quantize.restype = ctypes.c_int
    L.lrc_q4_apply.argtypes = [_vp, _vp, ctypes.c_int, _i64, _vp, _vp, _vp, _i64, ctypes.c_int, _vp, _i64, _vp, _i64,
                               _i64, _i64, _i64, ctypes.c_int, ctypes.c_int]
    L.lrc_q4_apply.restype = ctypes.c_int
    L.lrc_sample.argtypes = [_vp, _i64, _i64, _i64, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp]
    L.lrc_sample.restype = ctypes.c_int
    distill = [_vp, _i64, _i64, _i64, ctypes.c_int, _vp, _vp, _i64, ctypes.c_int, _vp, _vp, ctypes.c_double]
    L.lrc_distill.argtypes = distill + [_vp, _vp, _vp, _i64]
    L.lrc_distill.restype = ctypes.c_int
    L.lrc_distill_backward.argtypes = distill + [_vp, _vp, _vp, _i64]
    L.lrc_distill_backward.restype = ctypes.c_int
    L.lrc_q4_apply_e4m3.argtypes = [_vp, _vp, ctypes.c_int, _i64, _vp, _vp, _vp, _i64, ctypes.c_int, _vp, _i64, _vp, _vp,
                                    _i64, _i64, _i64, _i64, ctypes.c_int]
    L.lrc_q4_apply_e4m3.restype = ctypes.c_int
    L.lrc_rms_norm.argtypes = [_vp, _i64, _vp, _i64, _i64, _i64, ctypes.c_int, _vp, ctypes.c_int, ctypes.c_double, _vp,
                               _i64, _vp, _i64, ctypes.c_int, _vp, _vp]
    L.lrc_rms_norm.restype = ctypes.c_int
    L.lrc_rms_norm_backward.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i64, ctypes.c_int, _vp, ctypes.c_int, _vp, _i64,
                                        _vp, _i64, _vp]
    L.lrc_rms_norm_backward.restype = ctypes.c_int
    L.lrc_adapter_apply.argtypes = [_vp, _i64, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64, ctypes.c_int, _vp, _i64,
                                    _vp, _i64, _vp]
    L.lrc_adapter_apply.restype = ctypes.c_int
    L.lrc_adapter_backward.argtypes = [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                                       ctypes.c_int, _vp, _i64, _vp, _i64, _vp, _vp]
    L.lrc_adapter_backward.restype = ctypes.c_int
    L.lrc_verify.argtypes = [_vp, _i64, _i64, _vp, _i64, _i64, _i64, _i64, _i64, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp,
                             _vp, _vp]
    L.lrc_verify.restype = ctypes.c_int
    L.lrc_storage_bytes.argtypes = [_i64, _i64, _i64, ctypes.c_int]
    L.lrc_storage_bytes.restype = _i64
    L.lrc_tt_storage_bytes.argtypes = [ctypes.POINTER(_i64), ctypes.POINTER(_i64), ctypes.c_int, ctypes.c_int]
    L.lrc_tt_storage_bytes.restype = _i64
    L.lrc_set_stream.argtypes = [_vp]
    L.lrc_set_stream.restype = ctypes.c_int
    L.lrc_last_error.argtypes = []
    L.lrc_last_error.restype = ctypes.c_char_p
    L.lrc_shutdown.argtypes = []
    L.lrc_shutdown.restype = None
    L.lrc_version.argtypes = []
    L.lrc_version.restype = ctypes.c_int
    L.lrc_profile_enable.argtypes = [ctypes.c_int]
    L.lrc_profile_enable.restype = ctypes.c_int
    L.lrc_profile_filter.argtypes = [ctypes.c_char_p]
    L.lrc_profile_filter.restype = ctypes.c_int
    L.lrc_profile_reset.argtypes = []
    L.lrc_profile_reset.restype = None
    L.lrc_profile_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(_i64), ctypes.POINTER(ctypes.c_double)]
    L.lrc_profile_read.restype = ctypes.c_int
    L.lrc_profile_labels.argtypes = [ctypes.c_char_p, _i64]
    L.lrc_profile_labels.restype = _i64
    _lib = L
    return L


def header_symbols():
    """Function names declared in include/lrc.h."""
    with open(HEADER) as fh:
        text = fh.read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?[\w\s\*]*?\b(lrc_\w+)\s*\(", text, flags=re.M)))


def _check(rc: int):
    if rc < 0:
        raise LrcError(rc, lib().lrc_last_error().decode())
    return rc


# The small calls are bound by the host (a call of 10 us spends 7 in this
# file's checks when written carelessly), so the dtype table is built once and
# the current stream is read as a raw handle, without a Stream object
# (0.1 against 2.3 us).
_dtypes = None
_plain = None
_raw_stream = None


def _prec_of(t) -> int:
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = {torch.float64: FP64, torch.float32: FP32, torch.float16: FP16}
    p = _dtypes.get(t.dtype)
    if p is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return p


def _new(t, shape):
    """An uninitialised plain tensor of t's dtype on its device."""
    global _plain
    if _plain is None:
        import torch
        _plain = torch.Tensor
    if type(t) is _plain:
        return t.new_empty(shape)            # 2 us less than torch.empty
    import torch
    return torch.empty(shape, dtype=t.dtype, device=t.device)   # new_empty would keep a subclass


def _dev(*ts):
    for t in ts:
        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous (row-major)")


def _bind_stream(device):
    """Hands torch's current stream on the tensors' device to the library."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
    lib().lrc_set_stream(_raw_stream(device.index))


# ------------------------------------------------------------------ API ---

def storage_bytes(m: int, n: int, k: int, prec) -> int:
    p = PREC_NAMES.get(prec, prec)
    return _check(lib().lrc_storage_bytes(m, n, k, p))


def tt_storage_bytes(dims, ranks, prec) -> int:
    p = PREC_NAMES.get(prec, prec)
    d = len(dims)
    D = (_i64 * d)(*dims)
    R = (_i64 * (d + 1))(*ranks)
    return _check(lib().lrc_tt_storage_bytes(D, R, d, p))


def apply_path(m: int, n: int, k: int, batch: int, prec) -> int:
    p = PREC_NAMES.get(prec, prec)
    return _check(lib().lrc_matrix_apply_path(m, n, k, batch, p))


def set_apply_path(path: int):
    _check(lib().lrc_set_apply_path(path))


def _need(cond: bool, msg: str):
    if not cond:
        raise ValueError(msg)


def matrix_apply(U, s, V, X, Y=None):
    """Y = U diag(s) (V^T X): U (m x k), s (k), V (n x k), X (n x batch).
    A caller-supplied Y must be (m, batch), of U's dtype and on U's device."""
    prec = _prec_of(U)
    dt = U.dtype
    if s.dtype != dt or V.dtype != dt or X.dtype != dt:
        raise TypeError("all factors and the batch must share one dtype")
    _need(U.dim() == 2 and X.dim() == 2, "U and X must be matrices")
    m, k = U.shape
    n, b = X.shape
    if V.shape != (n, k) or s.shape != (k,):
        raise ValueError(f"shape mismatch: V {tuple(V.shape)} (want {(n, k)}), s {tuple(s.shape)} (want {(k,)})")
    if Y is not None:
        _need(tuple(Y.shape) == (m, b), f"Y has shape {tuple(Y.shape)}, want {(m, b)}")
        _need(Y.dtype == dt, f"Y has dtype {Y.dtype}, want {dt}")
    _dev(U, s, V, X)
    dev = U.device
    if Y is None:
        Y = _new(U, (m, b))
    else:
        _dev(Y)
    _need(s.device == dev and V.device == dev and X.device == dev and Y.device == dev,
          "all tensors must be on one device")
    _bind_stream(dev)
    rc = lib().lrc_matrix_apply(U.data_ptr(), s.data_ptr(), V.data_ptr(), X.data_ptr(), Y.data_ptr(), m, n, k, b,
                                prec)
    if rc < 0:
        _check(rc)
    return Y


def tt_shape(cores):
    dims = [int(c.shape[1]) for c in cores]
    ranks = [int(cores[0].shape[0])] + [int(c.shape[2]) for c in cores]
    return dims, ranks


def matrix_apply_noalloc(U, s, V, X, Y):
    """matrix_apply through the allocation-free entry point: Y (m x batch)
    must be supplied; the library's per-device scratch array holds the
    intermediate sums (calls overlapping on one device race on it)."""
    prec = _prec_of(U)
    for t in (s, V, X, Y):
        if t.dtype != U.dtype:
            raise TypeError("all factors, the batch and Y must share one dtype")
    _need(U.dim() == 2 and X.dim() == 2, "U and X must be matrices")
    m, k = U.shape
    n, b = X.shape
    _need(tuple(V.shape) == (n, k) and tuple(s.shape) == (k,), "shape mismatch")
    _need(tuple(Y.shape) == (m, b), f"Y has shape {tuple(Y.shape)}, want {(m, b)}")
    _dev(U, s, V, X, Y)
    _bind_stream(U.device)
    _check(lib().lrc_matrix_apply_noalloc(U.data_ptr(), s.data_ptr(), V.data_ptr(), X.data_ptr(), Y.data_ptr(),
                                          m, n, k, b, prec))
    return Y


def _check_train(cores):
    """Consistent TT cores: 3-D (r_{l-1}, n_l, r_l), adjacent ranks equal,
    boundary ranks 1, one dtype.  Returns their dims and ranks."""
    _need(len(cores) >= 1, "need at least one core")
    dt = cores[0].dtype
    dims, ranks = [], []
    for l, c in enumerate(cores):
        if c.dim() != 3:
            raise ValueError(f"core {l} must be 3-D (r_prev, n, r_next)")
        if c.dtype != dt:
            raise TypeError("all cores must share one dtype")
        r0, n, r1 = c.shape
        if l == 0:
            ranks.append(r0)
        elif r0 != ranks[l]:
            raise ValueError(f"core {l} starts with rank {r0}, core {l - 1} ends with {ranks[l]}")
        dims.append(n)
        ranks.append(r1)
    _need(ranks[0] == 1 and ranks[-1] == 1, "boundary ranks must be 1")
    return dims, ranks


def tt_reconstruct(cores, out=None):
    """Dense tensor (C order) from TT cores G_l of shape (r_{l-1}, n_l, r_l).
    A caller-supplied `out` must hold prod(dims) entries of the cores'
    dtype on their device."""
    prec = _prec_of(cores[0])
    dims, ranks = _check_train(cores)
    d = len(cores)
    if out is not None:
        _need(out.numel() == math.prod(dims), f"out has {out.numel()} entries, want {math.prod(dims)}")
        _need(out.dtype == cores[0].dtype, f"out has dtype {out.dtype}, want {cores[0].dtype}")
    _dev(*cores)
    dev = cores[0].device
    if out is None:
        out = _new(cores[0], dims)
    else:
        _dev(out)
    for c in cores:
        _need(c.device == dev and out.device == dev, "cores and out must be on one device")
    ptrs = (_vp * d)(*[c.data_ptr() for c in cores])
    D = (_i64 * d)(*dims)
    R = (_i64 * (d + 1))(*ranks)
    _bind_stream(dev)
    _check(lib().lrc_tt_reconstruct(ptrs, D, R, d, out.data_ptr(), prec))
    return out


def round_to(x, prec, out=None, count_overflow: bool = False):
    """Stored values of a float64 tensor: one round-to-nearest-even step to
    `prec` ("fp32" / "fp16", or a torch dtype).  Returns the rounded tensor,
    and with count_overflow=True also the number of finite values that
    became infinite (this waits for the result)."""
    import torch
    _dev(x)
    if x.dtype != torch.float64:
        raise TypeError("x must be float64")
    dt = {"fp64": torch.float64, "fp32": torch.float32, "fp16": torch.float16}.get(prec, prec)
    p = {torch.float64: FP64, torch.float32: FP32, torch.float16: FP16}[dt]
    if out is None:
        out = torch.empty(x.shape, dtype=dt, device=x.device)
    _dev(out)
    if out.dtype != dt or out.numel() != x.numel():
        raise ValueError("out must have the target dtype and x's size")
    _bind_stream(x.device)
    n = _i64(0)
    _check(lib().lrc_round(x.data_ptr(), out.data_ptr(), x.numel(), p, ctypes.byref(n) if count_overflow else None))
    return (out, int(n.value)) if count_overflow else out


def tt_left_orthogonalize(cores):
    """Left-orthogonal gauge of float64 TT cores (r_{l-1}, n_l, r_l), in
    place; returns the same list."""
    import torch
    _dev(*cores)
    for c in cores:
        if c.dtype != torch.float64:
            raise TypeError("the gauge takes float64 cores")
    dims, ranks = tt_shape(cores)
    d = len(cores)
    ptrs = (_vp * d)(*[c.data_ptr() for c in cores])
    D = (_i64 * d)(*dims)
    R = (_i64 * (d + 1))(*ranks)
    _bind_stream(cores[0].device)
    _check(lib().lrc_tt_left_orthogonalize(ptrs, D, R, d))
    return cores


def _quality(q: Quality) -> dict:
    return {f: getattr(q, f) for f, _ in Quality._fields_}


def band_quality(X, Xh, scale: float = 1.0) -> dict:
    """Quality of Xh (any storage dtype) against the float64 reference X,
    bands along the last axis (relative error, mean band PSNR, mean band
    SSIM variant, mean spectral angle)."""
    import torch
    _dev(X, Xh)
    if X.dtype != torch.float64 or X.shape != Xh.shape or X.dim() < 2:
        raise ValueError("X must be float64 with at least two axes, Xh of the same shape")
    B = int(X.shape[-1])
    _bind_stream(X.device)
    q = Quality()
    _check(lib().lrc_band_quality(X.data_ptr(), Xh.data_ptr(), X.numel() // B, B, _prec_of(Xh), float(scale),
                                  ctypes.byref(q)))
    return _quality(q)


def tt_quality(cores, X, scale: float = 1.0) -> dict:
    """Quality of the FP64 contraction of the stored cores (times scale)
    against the float64 reference X of the full tensor shape."""
    import torch
    _dev(*cores, X)
    if X.dtype != torch.float64:
        raise TypeError("X must be float64")
    dims, ranks = tt_shape(cores)
    if list(X.shape) != dims:
        raise ValueError("X must have the tensor's shape")
    d = len(cores)
    ptrs = (_vp * d)(*[c.data_ptr() for c in cores])
    D = (_i64 * d)(*dims)
    R = (_i64 * (d + 1))(*ranks)
    _bind_stream(X.device)
    q = Quality()
    _check(lib().lrc_tt_quality(ptrs, D, R, d, _prec_of(cores[0]), X.data_ptr(), float(scale), ctypes.byref(q)))
    return _quality(q)


def memory_matched_rank(dims, budget_bytes: int):
    """(R, capped rank vector) of the largest uniform FP64 TT rank within
    budget_bytes; (0, None) if rank 1 does not fit."""
    d = len(dims)
    D = (_i64 * d)(*dims)
    out = (_i64 * (d + 1))()
    R = _check(lib().lrc_tt_memory_matched_rank(D, d, int(budget_bytes), out))
    return (int(R), [int(v) for v in out]) if R > 0 else (0, None)


def rsvd(A, omega, k: int, power_iters: int = 0):
    """Rank-k randomized SVD of the float64 device matrix A (m x n) with the
    test vectors as the rows of omega (l x n): returns U (m x k), s (k),
    V (n x k), float64 on A's device, with U diag(s) V^T = U U^T A."""
    import torch
    _dev(A, omega)
    if A.dtype != torch.float64 or omega.dtype != torch.float64 or A.dim() != 2 or omega.dim() != 2:
        raise ValueError("A and omega must be float64 matrices")
    m, n = (int(x) for x in A.shape)
    l = int(omega.shape[0])
    if int(omega.shape[1]) != n:
        raise ValueError("omega must have n columns")
    A = A.contiguous()
    omega = omega.contiguous()
    U = torch.empty((m, k), dtype=torch.float64, device=A.device)
    s = torch.empty(k, dtype=torch.float64, device=A.device)
    V = torch.empty((n, k), dtype=torch.float64, device=A.device)
    _bind_stream(A.device)
    _check(lib().lrc_rsvd(A.data_ptr(), m, n, omega.data_ptr(), l, int(power_iters), int(k), U.data_ptr(),
                          s.data_ptr(), V.data_ptr()))
    return U, s, V


def tt_rsvd(T, ranks, omegas, power_iters: int = 0):
    """Randomized TT-SVD of the float64 device tensor T at TT ranks
    `ranks` (d-1 values), omegas[l] holding the test vectors of step l as
    rows.  Returns (cores, sigmas): float64 cores (r_{l-1}, n_l, r_l) and
    the kept singular values of every step."""
    import torch
    _dev(T, *omegas)
    if T.dtype != torch.float64 or any(o.dtype != torch.float64 for o in omegas):
        raise ValueError("T and the test matrices must be float64")
    dims = [int(x) for x in T.shape]
    d = len(dims)
    rk = [1] + [int(r) for r in ranks] + [1]
    if len(rk) != d + 1 or len(omegas) != d - 1:
        raise ValueError("need d-1 ranks and d-1 test matrices")
    T = T.contiguous()
    oms = [o.contiguous() for o in omegas]
    cores = [torch.empty((rk[l], dims[l], rk[l + 1]), dtype=torch.float64, device=T.device) for l in range(d)]
    sig = torch.empty(sum(rk[1:d]), dtype=torch.float64, device=T.device)
    D = (_i64 * d)(*dims)
    R = (_i64 * (d + 1))(*rk)
    S = (_i64 * (d - 1))(*[int(o.shape[0]) for o in oms])
    O = (_vp * (d - 1))(*[o.data_ptr() for o in oms])
    C = (_vp * d)(*[c.data_ptr() for c in cores])
    _bind_stream(T.device)
    _check(lib().lrc_tt_rsvd(T.data_ptr(), D, R, d, O, S, int(power_iters), C, sig.data_ptr()))
    sigmas, o = [], 0
    for r in rk[1:d]:
        sigmas.append(sig[o:o + r])
        o += r
    return cores, sigmas


# ---- compressed output head ----

_head_dtypes = None


def _head_prec(dtype) -> int:
    """FP32, FP16 or BF16 of an activation, logit, scale or factor dtype."""
    global _head_dtypes
    if _head_dtypes is None:
        import torch
        _head_dtypes = {torch.float32: FP32, torch.float16: FP16, torch.bfloat16: BF16}
    p = _head_dtypes.get(dtype)
    if p is None:
        raise TypeError(f"unsupported dtype {dtype}")
    return p


def _rows(t, name):
    """Pitch of a matrix whose rows are contiguous."""
    shape, (ld, step) = t.shape, t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return ld if shape[0] > 1 else max(ld, shape[1])


def _on(dev, **ts):
    """Every given tensor lives on the device `dev`, a GPU."""
    if dev.type != "cuda":
        raise ValueError("tensors must be on the GPU")
    for name, t in ts.items():
        if t is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the others on {dev}")


def q4_row_bytes(n: int) -> int:
    return _check(lib().lrc_q4_row_bytes(n))


def q4_storage_bytes(m: int, n: int, group: int, scale_prec) -> int:
    p = {"fp32": FP32, "fp16": FP16, "bf16": BF16}.get(scale_prec, scale_prec)
    return _check(lib().lrc_q4_storage_bytes(m, n, group, p))


def q4_quantize(W, group: int = 128, scale_dtype=None, values: bool = False, count_nonfinite: bool = False):
    """4-bit weights of the matrix W (m x n, float64, float32, float16 or
    bfloat16, contiguous rows): E2M1 codes (uint8, m x q4_row_bytes(n), two a
    byte) and scales (m x ceil(n / group), float16 unless scale_dtype says
    otherwise).  With values=True also the values they stand for, in W's
    dtype; with count_nonfinite=True also the number of groups that hold a
    NaN or an infinity or whose scale overflows (this waits for the result)."""
    import torch
    _need(W.dim() == 2, "W must be a matrix")
    prec = FP64 if W.dtype == torch.float64 else _head_prec(W.dtype)
    scale_dtype = scale_dtype or torch.float16
    sprec = _head_prec(scale_dtype)
    _need(group in (32, 64, 128, 256, 512), "group must be 32, 64, 128, 256 or 512")
    m, n = W.shape
    ld = _rows(W, "W")
    dev = W.device
    _on(dev)
    codes = torch.empty((m, (n + 31) // 32 * 16), dtype=torch.uint8, device=dev)
    scales = torch.empty((m, -(-n // group)), dtype=scale_dtype, device=dev)
    val = torch.empty((m, n), dtype=W.dtype, device=dev) if values else None
    bad = _i64(0)
    _bind_stream(dev)
    _check(lib().lrc_q4_quantize(W.data_ptr(), ld, m, n, group, prec, codes.data_ptr(), scales.data_ptr(), sprec,
                                 val.data_ptr() if values else None,
                                 ctypes.byref(bad) if count_nonfinite else None))
    out = (codes, scales) + ((val,) if values else ()) + ((int(bad.value),) if count_nonfinite else ())
    return out


def q4_apply(codes, scales, X, group: int = 128, factors=None, out_dtype=None, Y=None, x_scales=None):
    """Y = X W^T + [(X V) diag(s)] U^T: X (batch x n, float32, float16 or
    bfloat16, contiguous rows), W the m x n weights of `codes` and `scales`
    (q4_quantize), factors = (U, s, V) a rank-k compensation (U m x k, s k,
    V n x k, one dtype) or None.  Y (batch x m) is in out_dtype (X's unless
    given); a caller-supplied Y sets it.  X may be float8_e4m3fn with
    x_scales (float32, one factor per row, as rms_norm_e4m3 gives them): row b
    of the whole is times x_scales[b], and out_dtype is bfloat16 unless given:
    twice as fast in large batches as float16 and float32, whose sums are in
    float32 throughout."""
    _need(X.dim() == 2 and codes.dim() == 2 and scales.dim() == 2, "X, codes and scales must be matrices")
    _need(group in (32, 64, 128, 256, 512), "group must be 32, 64, 128, 256 or 512")
    b, n = X.shape
    m = codes.shape[0]
    if codes.dtype != _uint8():
        raise TypeError(f"codes have dtype {codes.dtype}, want uint8")
    if codes.shape[1] != (n + 31) // 32 * 16 or scales.shape != (m, -(-n // group)):
        raise ValueError(f"shape mismatch: codes {tuple(codes.shape)} (want {(m, (n + 31) // 32 * 16)}), "
                         f"scales {tuple(scales.shape)} (want {(m, -(-n // group))})")
    e4m3 = X.dtype == _e4m3_dtype()
    _need(e4m3 == (x_scales is not None), "x_scales belong to activations in float8_e4m3fn")
    if e4m3 and out_dtype is None:
        out_dtype = Y.dtype if Y is not None else _e4m3[1]
    prec, sprec = None if e4m3 else _head_prec(X.dtype), _head_prec(scales.dtype)
    ldx = _rows(X, "X")
    xs = _row_values(x_scales, "x_scales", b, _whole_dtypes()[2])
    k, fprec, ptrs = 0, 0, (None, None, None)
    dev = X.device
    if factors is not None:
        U, s, V = factors
        k = s.shape[0]
        if U.shape != (m, k) or V.shape != (n, k) or s.dim() != 1:
            raise ValueError(f"shape mismatch: U {tuple(U.shape)}, s {tuple(s.shape)}, V {tuple(V.shape)}")
        fprec = _head_prec(s.dtype)
        if U.dtype != s.dtype or V.dtype != s.dtype:
            raise TypeError("U, s and V must share one dtype")
        _dev(U, s, V)
        _on(dev, U=U, s=s, V=V)
        ptrs = (U.data_ptr(), s.data_ptr(), V.data_ptr())
    if Y is not None:
        _need(tuple(Y.shape) == (b, m), f"Y has shape {tuple(Y.shape)}, want {(b, m)}")
        _need(out_dtype is None or Y.dtype == out_dtype, f"Y has dtype {Y.dtype}, want {out_dtype}")
        ldy = _rows(Y, "Y")
        yprec = _head_prec(Y.dtype)
    else:
        yprec = prec if out_dtype is None else _head_prec(out_dtype)
    _dev(codes, scales)
    _on(dev, codes=codes, scales=scales, Y=Y)
    if Y is None:
        Y, ldy = _empty((b, m), out_dtype or X.dtype, dev), m
    if e4m3:
        _on(dev, x_scales=x_scales)
        _launch(dev, "lrc_q4_apply_e4m3", codes.data_ptr(), scales.data_ptr(), sprec, group, *ptrs, k, fprec,
                X.data_ptr(), ldx, xs, Y.data_ptr(), ldy, m, n, b, yprec)
        return Y
    _bind_stream(dev)
    rc = lib().lrc_q4_apply(codes.data_ptr(), scales.data_ptr(), sprec, group, *ptrs, k, fprec, X.data_ptr(), ldx,
                            Y.data_ptr(), ldy, m, n, b, prec, yprec)
    if rc < 0:
        _check(rc)
    return Y


def _empty(shape, dtype, device):
    import torch
    return torch.empty(shape, dtype=dtype, device=device)


_e4m3 = None


def _e4m3_dtype():
    """float8_e4m3fn, looked up once (with bfloat16 beside it)."""
    global _e4m3
    if _e4m3 is None:
        import torch
        _e4m3 = (torch.float8_e4m3fn, torch.bfloat16)
    return _e4m3[0]


_current = None


def _launch(dev, name, *args):
    """One call on torch's current stream of the tensors' device, which need
    not be the current one."""
    global _current
    if _current is None:
        import torch
        _current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    if _current() == dev.index:
        _bind_stream(dev)
        rc = getattr(lib(), name)(*args)
    else:
        import torch
        with torch.cuda.device(dev):
            _bind_stream(dev)
            rc = getattr(lib(), name)(*args)
    if rc < 0:
        _check(rc)


_whole = None


def _uint8():
    return _whole_dtypes()[0]


def _whole_dtypes():
    """(uint8, int64, float32), looked up once."""
    global _whole
    if _whole is None:
        import torch
        _whole = (torch.uint8, torch.int64, torch.float32)
    return _whole


def _row_values(t, name, rows, dtype):
    """Pointer of one value per row, or None."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, want {dtype}")
    if t.shape != (rows,) or not t.is_contiguous():
        raise ValueError(f"{name} must hold one contiguous value per row ({rows})")
    return t.data_ptr()


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, out=None):
    """One token index (int64) per row of logits (rows x vocab, float32,
    float16 or bfloat16, contiguous rows) from the uniform numbers u (float32,
    one per row).  temperature, top_p, min_p (float32) and top_k (int64) hold
    one value per row, or None: 1 and filters that are off.  A temperature
    that is not above 0 takes the largest logit; a row whose logits are all
    -infinity gives -1."""
    _need(logits.dim() == 2, "logits must be a matrix")
    rows, vocab = logits.shape
    prec = _head_prec(logits.dtype)
    ld = _rows(logits, "logits")
    _, i64, f32 = _whole_dtypes()
    pu = _row_values(u, "u", rows, f32)
    pt = _row_values(temperature, "temperature", rows, f32)
    pk = _row_values(top_k, "top_k", rows, i64)
    pp = _row_values(top_p, "top_p", rows, f32)
    pm = _row_values(min_p, "min_p", rows, f32)
    dev = logits.device
    _on(dev, u=u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, out=out)
    if out is None:
        out = _empty((rows,), i64, dev)
    po = _row_values(out, "out", rows, i64)
    _bind_stream(dev)
    rc = lib().lrc_sample(logits.data_ptr(), ld, rows, vocab, prec, pu, pt, pk, pp, pm, po)
    if rc < 0:
        _check(rc)
    return out


def _distill_args(logits, ids, top_logits, temperature, teacher_lse, weight):
    _need(logits.dim() == 2 and ids.dim() == 2, "logits, ids and top_logits must be matrices")
    rows, vocab = logits.shape
    _, i64, f32 = _whole_dtypes()
    if ids.dtype != i64:
        raise TypeError(f"ids have dtype {ids.dtype}, want {i64}")
    if ids.shape[0] != rows or top_logits.shape != ids.shape:
        raise ValueError(f"shape mismatch: ids {tuple(ids.shape)}, top_logits {tuple(top_logits.shape)}, {rows} rows")
    prec, tprec = _head_prec(logits.dtype), _head_prec(top_logits.dtype)
    lse = _row_values(teacher_lse, "teacher_lse", rows, f32)
    w = _row_values(weight, "weight", rows, f32)
    ld = _rows(logits, "logits")
    _dev(ids, top_logits)
    _on(logits.device, ids=ids, top_logits=top_logits, teacher_lse=teacher_lse, weight=weight)
    return (logits.data_ptr(), ld, rows, vocab, prec, ids.data_ptr(), top_logits.data_ptr(), ids.shape[1], tprec, lse, w,
            float(temperature))


def _grad_like(logits, grad):
    if grad is None:
        return _empty(tuple(logits.shape), logits.dtype, logits.device)
    _need(grad.shape == logits.shape and grad.dtype == logits.dtype, "grad must have the logits' shape and dtype")
    _on(logits.device, grad=grad)
    return grad


def distill(logits, ids, top_logits, temperature: float = 1.0, teacher_lse=None, weight=None, grad=None):
    """Distillation loss of every row (float32) and the gradient of their sum
    by the student's logits, in one pass: logits rows x vocab (float32,
    float16 or bfloat16, contiguous rows), ids (int64) and top_logits rows x K
    the teacher's named tokens (an id outside the vocabulary is an unused
    slot).  Without teacher_lse the teacher is renormalized over them; with it
    (float32, log-sum-exp of the teacher's logits / temperature) the rest of
    both distributions is one more class.  weight (float32) scales each row's
    loss; rows of weight 0 are not read.  grad may be the logits themselves."""
    args = _distill_args(logits, ids, top_logits, temperature, teacher_lse, weight)
    g = _grad_like(logits, grad)
    loss = _empty((args[2],), _whole_dtypes()[2], logits.device)
    _bind_stream(logits.device)
    _check(lib().lrc_distill(*args, loss.data_ptr(), None, g.data_ptr(), _rows(g, "grad")))
    return loss, g


def distill_forward(logits, ids, top_logits, temperature: float = 1.0, teacher_lse=None, weight=None):
    """The loss of distill alone, and the statistics (rows x 4, float32) that
    distill_backward takes."""
    args = _distill_args(logits, ids, top_logits, temperature, teacher_lse, weight)
    f32 = _whole_dtypes()[2]
    loss, stats = _empty((args[2],), f32, logits.device), _empty((args[2], 4), f32, logits.device)
    _bind_stream(logits.device)
    _check(lib().lrc_distill(*args, loss.data_ptr(), stats.data_ptr(), None, 0))
    return loss, stats


def distill_backward(logits, ids, top_logits, stats, dloss=None, temperature: float = 1.0, teacher_lse=None, weight=None,
                     grad=None):
    """Gradient of sum_i dloss_i loss_i by the logits, from the same inputs as
    distill_forward and the statistics that it gave (dloss float32, one per
    row, or None: 1).  grad may be the logits themselves."""
    args = _distill_args(logits, ids, top_logits, temperature, teacher_lse, weight)
    f32 = _whole_dtypes()[2]
    _need(stats.shape == (args[2], 4) and stats.dtype == f32, "stats must be float32, rows x 4")
    up = _row_values(dloss, "dloss", args[2], f32)
    _dev(stats)
    _on(logits.device, stats=stats, dloss=dloss)
    g = _grad_like(logits, grad)
    _bind_stream(logits.device)
    _check(lib().lrc_distill_backward(*args, stats.data_ptr(), up, g.data_ptr(), _rows(g, "grad")))
    return g


# ---- around the compressed projections ----

def _like(t, name, shape, dtype, dev):
    """A caller's output, or a new one: (tensor, pitch)."""
    if t is None:
        return _empty(shape, dtype, dev), shape[1]
    _need(tuple(t.shape) == tuple(shape) and t.dtype == dtype, f"{name} must be {tuple(shape)} of {dtype}")
    _on(dev, **{name: t})
    return t, _rows(t, name)


def _norm_args(x, weight, residual, eps, sum_out):
    _need(x.dim() == 2, "x must be a matrix")
    rows, n = x.shape
    prec = _head_prec(x.dtype)
    ldx = _rows(x, "x")
    dev = x.device
    wprec = 0
    if weight is not None:
        wprec = _head_prec(weight.dtype)
        _need(weight.shape == (n,) and weight.is_contiguous(), f"weight must hold {n} contiguous values")
    if residual is None:
        _need(sum_out is None, "sum belongs to a residual")
        _on(dev, weight=weight)
        return (x.data_ptr(), ldx, None, 0, rows, n, prec, weight.data_ptr() if weight is not None else None, wprec,
                float(eps), None, 0), x, dev
    _need(residual.shape == x.shape and residual.dtype == x.dtype, "residual must have x's shape and dtype")
    _on(dev, weight=weight, residual=residual)
    h, ldh = _like(sum_out, "sum", (rows, n), x.dtype, dev)
    return (x.data_ptr(), ldx, residual.data_ptr(), _rows(residual, "residual"), rows, n, prec,
            weight.data_ptr() if weight is not None else None, wprec, float(eps), h.data_ptr(), ldh), h, dev


def rms_norm(x, weight=None, residual=None, eps: float = 1e-6, stats: bool = False, out=None, sum=None):
    """Root-mean-square norm of the rows of h = x + residual (rounded to x's
    dtype; h = x without one): y = h (mean h^2 + eps)^(-1/2) weight.  x and
    residual rows x n (float32, float16 or bfloat16, contiguous rows), weight
    (n, any of the three) or None.  Returns (y, h), with stats=True also the
    inverse roots (rows, float32) that rms_norm_backward takes.  h without a
    residual is x itself; a caller-supplied `sum` receives it else, and may be
    the residual or x."""
    args, h, dev = _norm_args(x, weight, residual, eps, sum)
    rows, n, prec = args[4], args[5], args[6]
    y, ldy = _like(out, "out", (rows, n), x.dtype, dev)
    rstd = _empty((rows,), _whole_dtypes()[2], dev) if stats else None
    _launch(dev, "lrc_rms_norm", *args, y.data_ptr(), ldy, prec, None, rstd.data_ptr() if stats else None)
    return (y, h, rstd) if stats else (y, h)


def rms_norm_e4m3(x, weight=None, residual=None, eps: float = 1e-6, out=None, sum=None):
    """rms_norm with y in 8 bits: returns (codes, scales, h), codes (rows x n,
    float8_e4m3fn) the values nearest to the float32 quotients y / scale and
    scales (rows, float32) max |y| / 448 of each row, as q4_apply takes them."""
    args, h, dev = _norm_args(x, weight, residual, eps, sum)
    rows, n = args[4], args[5]
    y, ldy = _like(out, "out", (rows, n), _e4m3_dtype(), dev)
    scales = _empty((rows,), _whole_dtypes()[2], dev)
    _launch(dev, "lrc_rms_norm", *args, y.data_ptr(), ldy, E4M3, scales.data_ptr(), None)
    return y, scales, h


def rms_norm_backward(dy, h, weight, rstd, dsum=None, dx=None):
    """Gradient of rms_norm from dy (the gradient of y), h and rstd as it
    returned them: (dx, dweight), dx that of h (of x and of the residual
    alike) with dsum added, the gradient that reaches h by other ways, and
    dweight in weight's dtype (None without a weight).  dx may be dy or dsum."""
    _need(dy.dim() == 2 and h.shape == dy.shape and h.dtype == dy.dtype, "dy and h must be matrices of one shape and dtype")
    rows, n = dy.shape
    prec = _head_prec(dy.dtype)
    dev = dy.device
    lddy, ldh = _rows(dy, "dy"), _rows(h, "h")
    pr = _row_values(rstd, "rstd", rows, _whole_dtypes()[2])
    _need(pr is not None, "rstd must be given")
    pd, ldd = None, 0
    if dsum is not None:
        _need(dsum.shape == dy.shape and dsum.dtype == dy.dtype, "dsum must have dy's shape and dtype")
        pd, ldd = dsum.data_ptr(), _rows(dsum, "dsum")
    pw, wprec, dw = None, 0, None
    if weight is not None:
        wprec = _head_prec(weight.dtype)
        _need(weight.shape == (n,) and weight.is_contiguous(), f"weight must hold {n} contiguous values")
        pw = weight.data_ptr()
    _on(dev, h=h, weight=weight, rstd=rstd, dsum=dsum)
    if weight is not None:
        dw = _empty((n,), weight.dtype, dev)
    dx, ldx = _like(dx, "dx", (rows, n), dy.dtype, dev)
    _launch(dev, "lrc_rms_norm_backward", dy.data_ptr(), lddy, h.data_ptr(), ldh, pr, rows, n, prec, pw, wprec, pd, ldd,
            dx.data_ptr(), ldx, dw.data_ptr() if dw is not None else None)
    return dx, dw


def _adapter_args(A, B, ids, scale, rows, dtype, dev):
    """(m, n, k, count, prec, pointers of A, B, ids and scale)"""
    prec = _head_prec(dtype)
    _need(A.dim() == 3 and B.dim() == 3, "A and B must be count x k x n and count x m x k")
    count, k, n = A.shape
    m = B.shape[1]
    if B.shape != (count, m, k):
        raise ValueError(f"shape mismatch: A {tuple(A.shape)}, B {tuple(B.shape)}")
    _, i64, f32 = _whole_dtypes()
    if A.dtype != dtype or B.dtype != dtype:
        raise TypeError(f"A and B have dtype {A.dtype} and {B.dtype}, want {dtype}")
    pi = _row_values(ids, "ids", rows, i64)
    _need(pi is not None, "ids must be given")
    if scale is not None:
        if scale.dtype != f32:
            raise TypeError(f"scale has dtype {scale.dtype}, want {f32}")
        _need(scale.shape == (count,) and scale.is_contiguous(), f"scale must hold {count} contiguous values")
    _on(dev, A=A, B=B, ids=ids, scale=scale)
    _need(A.is_contiguous() and B.is_contiguous(), "tensors must be contiguous (row-major)")
    return m, n, k, count, prec, A.data_ptr(), B.data_ptr(), pi, scale.data_ptr() if scale is not None else None


def adapter_apply(X, A, B, ids, scale=None, base=None, hidden: bool = False, Y=None):
    """Low-rank adapters of many requests beside a shared projection:
    Y_i = base_i + scale_a (X_i A_a^T) B_a^T with a = ids_i (int64, one per
    row); rows whose id is outside [0, count) have none.  X rows x n (float32,
    float16 or bfloat16, contiguous rows), A count x k x n, B count x m x k,
    base (rows x m, what the shared projection gave) or None: 0, all of X's
    dtype, scale (count, float32) or None: 1.  Y may be base.  With
    hidden=True also X_i A_a^T (rows x k, float32), which adapter_backward
    takes."""
    _need(X.dim() == 2, "X must be a matrix")
    rows = X.shape[0]
    dev = X.device
    m, n, k, count, prec, pA, pB, pi, ps = _adapter_args(A, B, ids, scale, rows, X.dtype, dev)
    _need(X.shape[1] == n, f"X has {X.shape[1]} columns, A {n}")
    ldx = _rows(X, "X")
    pb, ldb = None, 0
    if base is not None:
        _need(base.shape == (rows, m) and base.dtype == X.dtype, f"base must be {(rows, m)} of {X.dtype}")
        _on(dev, base=base)
        pb, ldb = base.data_ptr(), _rows(base, "base")
    Y, ldy = _like(Y, "Y", (rows, m), X.dtype, dev)
    H = _empty((rows, k), _whole_dtypes()[2], dev) if hidden else None
    _launch(dev, "lrc_adapter_apply", X.data_ptr(), ldx, pA, pB, pi, ps, rows, m, n, k, count, prec, pb, ldb,
            Y.data_ptr(), ldy, H.data_ptr() if hidden else None)
    return (Y, H) if hidden else Y


def adapter_backward(dY, X, A, B, ids, hidden, scale=None, base=None, dX=None):
    """Gradients (dX, dA, dB) of adapter_apply from dY (rows x m) and the
    hidden values that it returned; base (rows x n, X's dtype) is added to dX,
    the shared projection's part of it (dX may be base).  base's own gradient
    is dY; adapters without rows get zeros."""
    _need(X.dim() == 2 and dY.dim() == 2, "X and dY must be matrices")
    rows = X.shape[0]
    dev = X.device
    m, n, k, count, prec, pA, pB, pi, ps = _adapter_args(A, B, ids, scale, rows, X.dtype, dev)
    _need(X.shape[1] == n, f"X has {X.shape[1]} columns, A {n}")
    _need(dY.shape == (rows, m) and dY.dtype == X.dtype, f"dY must be {(rows, m)} of {X.dtype}")
    _need(hidden.shape == (rows, k) and hidden.dtype == _whole_dtypes()[2] and hidden.is_contiguous(),
          f"hidden must be {(rows, k)} of float32, contiguous")
    ldx, lddy = _rows(X, "X"), _rows(dY, "dY")
    _on(dev, dY=dY, hidden=hidden, base=base)
    pb, ldb = None, 0
    if base is not None:
        _need(base.shape == (rows, n) and base.dtype == X.dtype, f"base must be {(rows, n)} of {X.dtype}")
        pb, ldb = base.data_ptr(), _rows(base, "base")
    dX, lddx = _like(dX, "dX", (rows, n), X.dtype, dev)
    dA, dB = _empty((count, k, n), X.dtype, dev), _empty((count, m, k), X.dtype, dev)
    _launch(dev, "lrc_adapter_backward", dY.data_ptr(), lddy, X.data_ptr(), ldx, pA, pB, pi, ps, hidden.data_ptr(), rows,
            m, n, k, count, prec, pb, ldb, dX.data_ptr(), lddx, dA.data_ptr(), dB.data_ptr())
    return dX, dA, dB


def _request_rows(t, name, requests, rows, vocab):
    """Pitches (of a row, of a request) of requests x rows x vocab logits."""
    _need(t.shape == (requests, rows, vocab), f"{name} has shape {tuple(t.shape)}, want {(requests, rows, vocab)}")
    lr, ld, step = t.stride()
    if step != 1 and vocab > 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    ld = ld if rows > 1 else vocab
    return ld, lr if requests > 1 else max(ld, vocab)


def verify(logits, drafts, u, draft_logits=None, temperature=None, top_k=None, top_p=None, min_p=None):
    """Drafted tokens checked against the target's logits so that the tokens
    follow the distribution that sample draws from: (tokens, accepted), tokens
    requests x (D + 1) (int64: the accepted drafts, one drawn token, then -1)
    and accepted (requests, int64).  logits requests x (D + 1) x vocab
    (float32, float16 or bfloat16, contiguous rows): row j behind the first j
    drafts; drafts requests x D (int64), one outside the vocabulary ends its
    request's; draft_logits requests x D x vocab what sample drew them from
    under the same parameters, or None: drafts that were certain; u requests x
    (D + 1) (float32) uniform numbers, the last for the drawn token;
    temperature, top_p, min_p (float32) and top_k (int64) one value per
    request, or None, as in sample."""
    _need(logits.dim() == 3 and drafts.dim() == 2, "logits must have three dimensions, drafts two")
    R, D = drafts.shape
    vocab = logits.shape[2]
    prec = _head_prec(logits.dtype)
    _, i64, f32 = _whole_dtypes()
    if drafts.dtype != i64 or u.dtype != f32:
        raise TypeError(f"drafts and u have dtype {drafts.dtype} and {u.dtype}, want {i64} and {f32}")
    ld, lr = _request_rows(logits, "logits", R, D + 1, vocab)
    _need(u.shape == (R, D + 1), f"u has shape {tuple(u.shape)}, want {(R, D + 1)}")
    _need(drafts.is_contiguous() and u.is_contiguous(), "drafts and u must be contiguous (row-major)")
    pq, ldq, lrq = None, 0, 0
    if draft_logits is not None:
        if draft_logits.dtype != logits.dtype:
            raise TypeError(f"draft_logits have dtype {draft_logits.dtype}, want {logits.dtype}")
        ldq, lrq = _request_rows(draft_logits, "draft_logits", R, D, vocab)
        pq = draft_logits.data_ptr()
    pt = _row_values(temperature, "temperature", R, f32)
    pk = _row_values(top_k, "top_k", R, i64)
    pp = _row_values(top_p, "top_p", R, f32)
    pm = _row_values(min_p, "min_p", R, f32)
    dev = logits.device
    _on(dev, drafts=drafts, u=u, draft_logits=draft_logits, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    tokens, accepted = _empty((R, D + 1), i64, dev), _empty((R,), i64, dev)
    _launch(dev, "lrc_verify", logits.data_ptr(), ld, lr, pq, ldq, lrq, R, D, vocab, prec, drafts.data_ptr(), u.data_ptr(),
            pt, pk, pp, pm, tokens.data_ptr(), accepted.data_ptr())
    return tokens, accepted


def _result(res: CertResult) -> dict:
    out = {f: getattr(res, f) for f, _ in CertResult._fields_}
    for f in ("certified", "acc_nonincrease", "acc_win", "mem_win", "practical_win"):
        out[f] = bool(out[f])
    return out


def certify_matrix(sigma, U, s, V, Uh, sh, Vh, k: int, A=None) -> dict:
    """Matrix certificate for base rank k (FP64) vs rank k+1 stored as
    (Uh, sh, Vh).  sigma: host sequence of all min(m, n) singular values;
    U (m x k+1), s (k+1), V (n x k+1) float64; Uh, sh, Vh the same shapes
    in float32 or float16; A (m x n, float64) or None."""
    import numpy as np
    import torch
    sig = np.ascontiguousarray(np.asarray(sigma, dtype=np.float64))
    _need(U.dim() == 2 and V.dim() == 2, "U and V must be matrices")
    m, n, r = int(U.shape[0]), int(V.shape[0]), int(k) + 1
    _need(int(k) >= 1 and tuple(U.shape) == (m, r) and tuple(V.shape) == (n, r) and tuple(s.shape) == (r,),
          f"FP64 factors must have k + 1 = {r} columns: U {tuple(U.shape)}, s {tuple(s.shape)}, V {tuple(V.shape)}")
    for name, t in (("U", U), ("s", s), ("V", V)):
        if t.dtype != torch.float64:
            raise TypeError(f"{name} must be float64")
    for name, t, ref in (("Uh", Uh, U), ("sh", sh, s), ("Vh", Vh, V)):
        _need(tuple(t.shape) == tuple(ref.shape), f"{name} has shape {tuple(t.shape)}, want {tuple(ref.shape)}")
        if t.dtype != Uh.dtype or t.dtype not in (torch.float16, torch.float32, torch.float64):
            raise TypeError("Uh, sh, Vh must share one storage dtype")
    _need(sig.ndim == 1 and sig.size == min(m, n), f"sigma must hold all min(m, n) = {min(m, n)} singular values")
    if A is not None:
        _need(tuple(A.shape) == (m, n), f"A has shape {tuple(A.shape)}, want {(m, n)}")
        if A.dtype != torch.float64:
            raise TypeError("A must be float64")
    _dev(U, s, V, Uh, sh, Vh)
    if A is not None:
        _dev(A)
    a = CertArgs()
    a.kind = CERT_MATRIX
    a.prec = _prec_of(Uh)
    a.m, a.n, a.k = m, n, int(k)
    a.sigma = sig.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
    a.n_sigma = len(sig)
    a.U, a.s, a.V = U.data_ptr(), s.data_ptr(), V.data_ptr()
    a.Uh, a.sh, a.Vh = Uh.data_ptr(), sh.data_ptr(), Vh.data_ptr()
    a.A = A.data_ptr() if A is not None else None
    res = CertResult()
    _bind_stream(U.device)
    _check(lib().lrc_certify(ctypes.byref(a), ctypes.byref(res)))
    return _result(res)


def certify_tt(T, base_cores, aug_cores, aug_cores_h) -> dict:
    """TT certificate: T dense FP64 of the trains' shape; FP64 base and
    augmented cores; the augmented cores as stored (FP32 or FP16), of the
    augmented cores' shapes."""
    import torch
    d = len(base_cores)
    _need(len(aug_cores) == d and len(aug_cores_h) == d, "the three trains must have the same number of cores")
    for cs in (base_cores, aug_cores, aug_cores_h):
        _check_train(cs)
    for cs in (base_cores, aug_cores):
        if cs[0].dtype != torch.float64:
            raise TypeError("base and augmented cores must be float64")
    dims, rb = tt_shape(base_cores)
    dims_a, ra = tt_shape(aug_cores)
    _need(dims_a == dims, f"augmented train has dims {dims_a}, base {dims}")
    for l in range(d):
        _need(tuple(aug_cores_h[l].shape) == tuple(aug_cores[l].shape),
              f"stored core {l} has shape {tuple(aug_cores_h[l].shape)}, want {tuple(aug_cores[l].shape)}")
    _need(T.numel() == math.prod(dims), f"T has {T.numel()} entries, want {math.prod(dims)}")
    if T.dtype != torch.float64:
        raise TypeError("T must be float64")
    _dev(T, *base_cores, *aug_cores, *aug_cores_h)
    a = CertArgs()
    a.kind = CERT_TT
    a.prec = _prec_of(aug_cores_h[0])
    a.d = d
    D = (_i64 * d)(*dims)
    RB = (_i64 * (d + 1))(*rb)
    RA = (_i64 * (d + 1))(*ra)
    PB = (_vp * d)(*[c.data_ptr() for c in base_cores])
    PA = (_vp * d)(*[c.data_ptr() for c in aug_cores])
    PH = (_vp * d)(*[c.data_ptr() for c in aug_cores_h])
    a.dims, a.ranks_base, a.ranks_aug = D, RB, RA
    a.cores_base, a.cores_aug, a.cores_aug_h = PB, PA, PH
    a.T = T.data_ptr()
    res = CertResult()
    _bind_stream(T.device)
    _check(lib().lrc_certify(ctypes.byref(a), ctypes.byref(res)))
    return _result(res)


def profile_enable(on: bool = True):
    _check(lib().lrc_profile_enable(1 if on else 0))


def profile_filter(label=None):
    """Time only launches labelled `label` (None: every launch)."""
    _check(lib().lrc_profile_filter(label.encode() if label else None))


def profile_reset():
    lib().lrc_profile_reset()


def mfma_ceiling(prec: str) -> float:
    """Measured matrix-core ceiling (TFLOP/s) of the kernels' MFMA
    instruction for prec ('fp64', 'fp32' or 'fp16') on the current device."""
    codes = {"fp64": 0, "fp32": 1, "fp16": 2}
    if prec not in codes:
        raise ValueError(f"prec must be one of {sorted(codes)}")
    out = ctypes.c_double()
    _check(lib().lrc_mfma_ceiling(codes[prec], ctypes.byref(out)))
    return float(out.value)


def profile_read() -> dict:
    """{kernel label: (launches, total milliseconds)} for every label seen."""
    L = lib()
    n = _check(L.lrc_profile_labels(None, 0))
    buf = ctypes.create_string_buffer(n + 1)
    L.lrc_profile_labels(buf, n + 1)
    out = {}
    for lab in filter(None, buf.value.decode().split(",")):
        cnt, ms = _i64(), ctypes.c_double()
        _check(L.lrc_profile_read(lab.encode(), ctypes.byref(cnt), ctypes.byref(ms)))
        out[lab] = (cnt.value, ms.value)
    return out


def shutdown():
    lib().lrc_shutdown()
