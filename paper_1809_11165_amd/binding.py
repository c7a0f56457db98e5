"""ctypes binding over libbbmm.so -- argument marshalling only.

Every function mirrors one entry point of include/bbmm.h under the same name.  Device
arrays are torch CUDA (HIP) tensors; PyTorch is used only to own device memory and to
provide the stream.  There is no fallback: if the shared library is missing or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from dataclasses import dataclass, field
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbbmm.so")

KERNEL_RBF, KERNEL_MATERN52 = 0, 1
MODE_MATERIALISED, MODE_ONTHEFLY, MODE_SGPR = 0, 1, 2
TYPE_F32, TYPE_F16, TYPE_BF16 = 0, 1, 2
OK, EINVAL, ENOMEM, ENOTPD, ENONFINITE, EHIP, ENOCONV = 0, 1, 2, 3, 4, 5, 6
MAX_ITERS = 256

EXPORTS = [
    "bbmm_create", "bbmm_destroy", "bbmm_last_error", "bbmm_tune", "bbmm_mm_timing", "bbmm_loop_graph_stats",
    "bbmm_solve_logdet_grad",
    "bbmm_setup", "bbmm_build_khat", "bbmm_khat_block", "bbmm_sgpr_build", "bbmm_sgpr_root_rows",
    "bbmm_kernel_mm", "bbmm_pivoted_cholesky",
    "bbmm_precond_setup", "bbmm_precond_solve", "bbmm_make_probes", "bbmm_mbcg",
    "bbmm_tridiag_eig_batched", "bbmm_tridiag_eig_batched_noalloc", "bbmm_slq_logdet", "bbmm_slq_from_coeffs", "bbmm_dk_traces",
    "bbmm_predict_mean", "bbmm_predict_var",
    "bbmm_attend_workspace", "bbmm_attend", "bbmm_attend_grad",
    "bbmm_bucket_bias", "bbmm_bucket_bias_workspace", "bbmm_bucket_bias_grad",
]


class BbmmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("bbmm error %d: %s" % (code, msg))
        self.code = code


class _Problem(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("mode", C.c_int32),
                ("n", C.c_int64), ("d", C.c_int64), ("t", C.c_int64), ("k", C.c_int64),
                ("max_iters", C.c_int64), ("tol", C.c_double),
                ("n_lengthscale", C.c_int64), ("lengthscale", C.POINTER(C.c_double)),
                ("outputscale", C.c_double), ("noise", C.c_double),
                ("X", C.c_void_p), ("y", C.c_void_p), ("E1", C.c_void_p), ("E2", C.c_void_p),
                ("m", C.c_int64), ("Uind", C.c_void_p), ("jitter_rel", C.c_double),
                ("pivots_in", C.POINTER(C.c_int64)), ("u0_init", C.c_void_p)]


class _Result(C.Structure):
    _fields_ = [("u0", C.c_void_p), ("U", C.c_void_p),
                ("logdet", C.c_double), ("logdet_precond", C.c_double), ("yKinvy", C.c_double),
                ("nlml", C.c_double),
                ("trace", C.POINTER(C.c_double)), ("quad", C.POINTER(C.c_double)),
                ("grad_nlml", C.POINTER(C.c_double)),
                ("iters_run", C.c_int64), ("rank", C.c_int64),
                ("alpha", C.POINTER(C.c_double)), ("beta", C.POINTER(C.c_double)),
                ("resid", C.POINTER(C.c_double)), ("pivots", C.POINTER(C.c_int64)),
                ("slq_terms", C.POINTER(C.c_double))]


class _Attention(C.Structure):
    _fields_ = [("type", C.c_int32), ("two_sided", C.c_int32),
                ("batch", C.c_int64), ("heads", C.c_int64), ("kv_heads", C.c_int64), ("nq", C.c_int64),
                ("nk", C.c_int64), ("d", C.c_int64), ("dv", C.c_int64), ("scale", C.c_double),
                ("Q", C.c_void_p), ("K", C.c_void_p), ("V", C.c_void_p),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("q_len", C.c_void_p), ("k_len", C.c_void_p), ("key_mask", C.c_void_p), ("table", C.c_void_p),
                ("n_edges", C.c_int64), ("edges", C.POINTER(C.c_int32)), ("q_start", C.c_void_p)]


_lib = None


def load_library() -> C.CDLL:
    """Loads libbbmm.so; raises if it has not been built (python -m paper_1809_11165_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError("%s not found: build it with `python -m paper_1809_11165_amd.build`"
                                % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    for name in EXPORTS:
        getattr(lib, name)            # AttributeError if a declared symbol is missing
    lib.bbmm_last_error.restype = C.c_char_p
    lib.bbmm_last_error.argtypes = [C.c_void_p]
    lib.bbmm_create.argtypes = [C.POINTER(C.c_void_p), C.c_int, C.c_void_p]
    lib.bbmm_destroy.argtypes = [C.c_void_p]
    lib.bbmm_tune.argtypes = [C.c_void_p, C.c_char_p, C.c_int64]
    lib.bbmm_mm_timing.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                   C.POINTER(C.c_int64)]
    lib.bbmm_loop_graph_stats.argtypes = [C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    lib.bbmm_solve_logdet_grad.argtypes = [C.c_void_p, C.POINTER(_Problem), C.POINTER(_Result)]
    lib.bbmm_setup.argtypes = [C.c_void_p, C.POINTER(_Problem)]
    lib.bbmm_build_khat.argtypes = [C.c_void_p]
    lib.bbmm_khat_block.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_void_p]
    lib.bbmm_sgpr_build.argtypes = [C.c_void_p]
    lib.bbmm_sgpr_root_rows.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p]
    lib.bbmm_kernel_mm.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
    lib.bbmm_pivoted_cholesky.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int64),
                                          C.POINTER(C.c_int64)]
    lib.bbmm_precond_setup.argtypes = [C.c_void_p, C.POINTER(C.c_double)]
    lib.bbmm_precond_solve.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    lib.bbmm_make_probes.argtypes = [C.c_void_p, C.c_void_p]
    lib.bbmm_mbcg.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                              C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double),
                              C.POINTER(C.c_int64)]
    lib.bbmm_tridiag_eig_batched.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                             C.c_int64, C.c_int64, C.POINTER(C.c_double),
                                             C.POINTER(C.c_double)]
    lib.bbmm_tridiag_eig_batched_noalloc.argtypes = lib.bbmm_tridiag_eig_batched.argtypes
    lib.bbmm_slq_logdet.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.bbmm_slq_from_coeffs.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                         C.POINTER(C.c_double), C.POINTER(C.c_int64), C.c_int64, C.c_int64,
                                         C.c_double, C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.bbmm_dk_traces.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_double),
                                   C.POINTER(C.c_double)]
    lib.bbmm_predict_mean.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
    lib.bbmm_predict_var.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                                     C.POINTER(C.c_int64), C.POINTER(C.c_double)]
    lib.bbmm_attend_workspace.argtypes = [C.c_void_p, C.POINTER(_Attention), C.c_int32, C.POINTER(C.c_int64)]
    lib.bbmm_attend.argtypes = [C.c_void_p, C.POINTER(_Attention), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64]
    lib.bbmm_attend_grad.argtypes = [C.c_void_p, C.POINTER(_Attention), C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.POINTER(C.c_int64), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_int64]
    lib.bbmm_bucket_bias.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int64,
                                     C.POINTER(C.c_int32), C.c_int32, C.c_int64, C.c_void_p]
    lib.bbmm_bucket_bias_workspace.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_int64,
                                               C.c_int32, C.POINTER(C.c_int64)]
    lib.bbmm_bucket_bias_grad.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int64,
                                          C.c_int64, C.POINTER(C.c_int32), C.c_int32, C.c_int64, C.c_void_p, C.c_void_p,
                                          C.c_int64]
    _lib = lib
    return lib


def _dptr(a):
    return C.c_void_p(a.ctypes.data) if isinstance(a, np.ndarray) else C.c_void_p(a.data_ptr())


def _dbl(a: np.ndarray):
    return a.ctypes.data_as(C.POINTER(C.c_double))


def _check_dev(tensor, shape, name):
    import torch
    if not (isinstance(tensor, torch.Tensor) and tensor.is_cuda and tensor.dtype == torch.float32
            and tensor.is_contiguous()):
        raise TypeError("%s must be a contiguous float32 device tensor" % name)
    if tuple(tensor.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(tensor.shape), tuple(shape)))


@dataclass
class Problem:
    """Host description of one inference problem; X, y, E1, E2 are device tensors."""
    kernel: int
    mode: int
    X: "object"
    y: "object"
    lengthscale: np.ndarray
    outputscale: float
    noise: float
    E1: "object"
    E2: "object"
    k: int
    max_iters: int
    tol: float = 0.0
    Uind: "object" = None           # SGPR only: m x d device tensor of inducing inputs
    jitter_rel: float = 0.0         # SGPR only
    pivots_in: Optional[np.ndarray] = None   # replay this pivot order instead of the greedy rule
    u0_init: "object" = None                 # n device floats: warm start of the y column
    _keep: list = field(default_factory=list, repr=False)

    def to_c(self) -> _Problem:
        n, d = self.X.shape
        t = self.E2.shape[1]
        ls = np.ascontiguousarray(np.atleast_1d(self.lengthscale), dtype=np.float64)
        _check_dev(self.X, (n, d), "X")
        _check_dev(self.y, (n,), "y")
        _check_dev(self.E2, (n, t), "E2")
        if self.k > 0:
            _check_dev(self.E1, (self.k, t), "E1")
        self._keep = [ls]
        p = _Problem()
        p.kernel, p.mode = int(self.kernel), int(self.mode)
        p.n, p.d, p.t, p.k, p.max_iters = n, d, t, int(self.k), int(self.max_iters)
        p.tol = float(self.tol)
        p.n_lengthscale = ls.shape[0]
        p.lengthscale = _dbl(ls)
        p.outputscale, p.noise = float(self.outputscale), float(self.noise)
        p.X, p.y = self.X.data_ptr(), self.y.data_ptr()
        p.E1 = self.E1.data_ptr() if self.k > 0 else None
        p.E2 = self.E2.data_ptr()
        p.m, p.Uind, p.jitter_rel = 0, None, 0.0
        p.u0_init = None
        if self.u0_init is not None:
            _check_dev(self.u0_init, (n,), "u0_init")
            p.u0_init = self.u0_init.data_ptr()
        p.pivots_in = None
        if self.pivots_in is not None:
            piv = np.ascontiguousarray(self.pivots_in, dtype=np.int64)
            if piv.shape != (int(self.k),):
                raise ValueError("pivots_in must have k entries")
            self._keep.append(piv)
            p.pivots_in = piv.ctypes.data_as(C.POINTER(C.c_int64))
        if self.mode == MODE_SGPR:
            if self.Uind is None:
                raise ValueError("an SGPR problem needs Uind")
            _check_dev(self.Uind, (self.Uind.shape[0], d), "Uind")
            p.m, p.Uind, p.jitter_rel = int(self.Uind.shape[0]), self.Uind.data_ptr(), float(self.jitter_rel)
        return p


_codes = {}


def _type_of(tensor, name):
    """The library's code of a tensor's type."""
    if not _codes:
        import torch
        _codes.update({torch.float32: TYPE_F32, torch.float16: TYPE_F16, torch.bfloat16: TYPE_BF16})
    code = _codes.get(getattr(tensor, "dtype", None))
    if code is None:
        raise TypeError("%s must be a float32, float16 or bfloat16 tensor" % name)
    return code


def _check_same(tensor, shape, dtype, device, name, dense=True):
    """A tensor of this shape, type and device; dense, or with its last dimension contiguous.  (The first line is the
    usual way through: a few tenths of a microsecond of a call's ten.)"""
    try:
        if (tensor.dtype is dtype and tensor.shape == shape and tensor.device == device
                and (tensor.is_contiguous() or (not dense and tensor.stride(-1) == 1))):
            return
    except AttributeError:
        raise TypeError("%s must be a tensor of type %s" % (name, dtype)) from None
    if tensor.dtype is not dtype:
        raise TypeError("%s must be a tensor of type %s" % (name, dtype))
    if tensor.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, tensor.device, device))
    if tensor.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(tensor.shape), tuple(shape)))
    if dense:
        raise ValueError("%s must be contiguous" % name)
    if shape[-1] > 1 and tensor.numel():
        raise ValueError("the last dimension of %s must be contiguous" % name)


def bucket_edges(num_buckets: int, max_distance: int, two_sided: bool = True):
    """Edges of the usual buckets: unit steps up to half of a side's buckets, then equal steps of the logarithm of which the one behind
    the last edge would stand at max_distance (32 two-sided buckets and 128: the last edge is 91).  An edge is the first
    whole distance at or beyond its step, found in whole numbers (x^n against powers), so nothing is rounded at a border.  Edges
    ascend: of steps that fall on the same distance (32 one-sided buckets with 32 or 33, 64 with 64 to 70) the later ones move up by
    one, where the usual buckets leave one empty; such a table has no edges here that give its buckets."""
    side = num_buckets // 2 if two_sided else num_buckets
    if side < 1 or (two_sided and num_buckets % 2) or max_distance < 1:
        raise ValueError("num_buckets must be positive (even when two_sided) and max_distance at least 1")
    near = max(1, side // 2)
    far = max(int(max_distance), near + 1)
    n = side - near
    edges = list(range(1, near + 1))
    for k in range(1, n):
        want = near ** (n - k) * far ** k
        lo, hi = edges[-1] + 1, max(far, edges[-1] + 1)
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (lo, mid) if mid ** n >= want else (mid + 1, hi)
        edges.append(lo)
    return edges[:side - 1]


def _edges(edges):
    """Edges as the C array that a call takes (their range and order are checked by the library)."""
    try:
        e = array("i", edges if edges is not None else ())
    except OverflowError:
        raise ValueError("bucket edges must ascend within [1, 1024]") from None
    return (C.c_int32 * len(e)).from_buffer(e) if e else (C.c_int32 * 0)()


def _int64(x):
    """A whole number for an int64 argument: beyond that type, its ends (which the library refuses), not what is left of its bits."""
    return min(max(int(x), -2 ** 63), 2 ** 63 - 1)


@dataclass
class Attention:
    """One attention call (see include/bbmm.h, "Attention").  Q (batch, nq, heads, d), K (batch, nk, kv_heads, d), V (batch,
    nk, kv_heads, dv): device tensors of one type, any strides with the last dimension contiguous.  scale: default
    d^-1/2.  q_len, k_len: int32 (batch,); key_mask: bool or uint8 (batch, nk), true takes part; table: (heads, buckets)
    of Q's type with edges (see bucket_edges); q_start: int64 (batch,).  The calls record no graph of gradients: inputs that require
    grad are refused outside torch.no_grad() (a torch.autograd.Function with bbmm_attend_grad as its backward runs so)."""
    Q: "object"
    K: "object"
    V: "object"
    scale: Optional[float] = None
    q_len: "object" = None
    k_len: "object" = None
    key_mask: "object" = None
    table: "object" = None
    edges: "object" = None
    two_sided: bool = True
    q_start: "object" = None

    def tensors(self):
        return [t for t in (self.Q, self.K, self.V, self.q_len, self.k_len, self.key_mask, self.table, self.q_start)
                if t is not None]

    def to_c(self, device) -> _Attention:
        Q, K, V, table = self.Q, self.K, self.V, self.table
        code, t = _type_of(Q, "Q"), Q.dtype
        try:
            b, nq, h, d = Q.shape
            _, nk, hk, dv = V.shape
            _, _, _, _ = K.shape
        except ValueError:
            raise ValueError("Q, K and V must have four dimensions (batch, row, head, feature)") from None
        except AttributeError:
            raise TypeError("Q, K and V must be tensors") from None
        _check_same(Q, (b, nq, h, d), t, device, "Q", dense=False)
        _check_same(K, (b, nk, hk, d), t, device, "K", dense=False)
        _check_same(V, (b, nk, hk, dv), t, device, "V", dense=False)
        two, n, edges = bool(self.two_sided), 0, None
        if table is not None:
            edges = _edges(self.edges)
            n = len(edges)
            _check_same(table, (h, 2 * n + 2 if two else n + 1), t, device, "table")
        elif self.edges is not None:
            raise ValueError("edges without a table")
        a = _Attention(code, two, b, h, hk, nq, nk, d, dv, max(d, 1) ** -0.5 if self.scale is None else self.scale, Q.data_ptr(),
                       K.data_ptr(), V.data_ptr(), Q.stride()[:3], K.stride()[:3], V.stride()[:3])
        if table is not None:
            a.table, a.n_edges, a.edges = table.data_ptr(), n, edges
        if self.q_len is not None or self.k_len is not None or self.key_mask is not None or self.q_start is not None:
            import torch
            if self.q_len is not None:
                _check_same(self.q_len, (b,), torch.int32, device, "q_len")
                a.q_len = self.q_len.data_ptr()
            if self.k_len is not None:
                _check_same(self.k_len, (b,), torch.int32, device, "k_len")
                a.k_len = self.k_len.data_ptr()
            if self.key_mask is not None:
                kind = torch.uint8 if getattr(self.key_mask, "dtype", None) == torch.uint8 else torch.bool
                _check_same(self.key_mask, (b, nk), kind, device, "key_mask")
                a.key_mask = self.key_mask.data_ptr()
            if self.q_start is not None:
                _check_same(self.q_start, (b,), torch.int64, device, "q_start")
                a.q_start = self.q_start.data_ptr()
        return a


@dataclass
class Result:
    u0: "object"
    U: "object"
    logdet: float
    logdet_precond: float
    yKinvy: float
    nlml: float
    trace: np.ndarray
    quad: np.ndarray
    grad_nlml: np.ndarray
    iters_run: int
    rank: int
    alpha: np.ndarray
    beta: np.ndarray
    resid: np.ndarray
    pivots: np.ndarray
    slq_terms: np.ndarray
    estimator_rel_err: float = float("nan")   # filled by tests only


class Context:
    """Owns one bbmm_ctx bound to the current torch device and stream."""

    def __init__(self, device: int = 0, stream=None):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the BBMM path only runs on the HIP library")
        self.lib = load_library()
        self.torch = torch
        self.device = torch.device("cuda", device)
        self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._raw_stream = self._stream.cuda_stream
        handle = C.c_void_p()
        rc = self.lib.bbmm_create(C.byref(handle), device, C.c_void_p(self._stream.cuda_stream))
        if rc != OK:
            raise BbmmError(rc, "bbmm_create failed")
        self.h = handle
        self._prob = None

    def close(self):
        if getattr(self, "h", None):
            self.lib.bbmm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ck(self, rc: int):
        if rc != OK:
            raise BbmmError(rc, self.lib.bbmm_last_error(self.h).decode())

    def _empty(self, *shape):
        return self.torch.empty(*shape, dtype=self.torch.float32, device=self.device)

    # ---- entry points (names follow include/bbmm.h) ------------------------------------
    def bbmm_tune(self, key: str, value: int):
        self._ck(self.lib.bbmm_tune(self.h, key.encode(), int(value)))

    def bbmm_mm_timing(self):
        """(average ms per K_hat.M launch, total ms, launches) of the last timed mBCG run."""
        avg, tot, cnt = C.c_double(0.0), C.c_double(0.0), C.c_int64(0)
        self._ck(self.lib.bbmm_mm_timing(self.h, C.byref(avg), C.byref(tot), C.byref(cnt)))
        return float(avg.value), float(tot.value), int(cnt.value)

    def bbmm_loop_graph_stats(self):
        """(graphs recorded, graphs replayed) by this context so far."""
        cap, rep = C.c_int64(0), C.c_int64(0)
        self._ck(self.lib.bbmm_loop_graph_stats(self.h, C.byref(cap), C.byref(rep)))
        return int(cap.value), int(rep.value)

    def bbmm_solve_logdet_grad(self, prob: Problem, want_U: bool = True) -> Result:
        p = prob.to_c()
        n, t, k, it = p.n, p.t, p.k, p.max_iters
        H = p.n_lengthscale + 2
        u0 = self._empty(n)
        U = self._empty(n, t + 1) if want_U else None
        trace, quad, grad = np.zeros(H), np.zeros(H), np.zeros(H)
        alpha, beta, resid = (np.zeros((it, t + 1)) for _ in range(3))
        pivots = np.full(max(k, 1), -1, dtype=np.int64)
        slq = np.zeros(t)
        r = _Result()
        r.u0 = u0.data_ptr()
        r.U = U.data_ptr() if want_U else None
        r.trace, r.quad, r.grad_nlml = _dbl(trace), _dbl(quad), _dbl(grad)
        r.alpha, r.beta, r.resid = _dbl(alpha), _dbl(beta), _dbl(resid)
        r.pivots = pivots.ctypes.data_as(C.POINTER(C.c_int64))
        r.slq_terms = _dbl(slq)
        self._ck(self.lib.bbmm_solve_logdet_grad(self.h, C.byref(p), C.byref(r)))
        self._prob = prob
        self._shape = (int(p.n), int(p.d), int(p.t), int(p.k), int(p.max_iters), int(p.n_lengthscale))
        return Result(u0=u0, U=U, logdet=r.logdet, logdet_precond=r.logdet_precond, yKinvy=r.yKinvy,
                      nlml=r.nlml, trace=trace, quad=quad, grad_nlml=grad, iters_run=int(r.iters_run),
                      rank=int(r.rank), alpha=alpha, beta=beta, resid=resid, pivots=pivots[:k],
                      slq_terms=slq)

    def bbmm_setup(self, prob: Problem):
        p = prob.to_c()
        self._ck(self.lib.bbmm_setup(self.h, C.byref(p)))
        self._prob = prob
        self._shape = (int(p.n), int(p.d), int(p.t), int(p.k), int(p.max_iters), int(p.n_lengthscale))

    def bbmm_build_khat(self):
        self._ck(self.lib.bbmm_build_khat(self.h))

    def bbmm_khat_block(self, row0: int, nrows: int, col0: int, ncols: int):
        out = self._empty(nrows, ncols)
        self._ck(self.lib.bbmm_khat_block(self.h, row0, nrows, col0, ncols, _dptr(out)))
        return out

    def bbmm_sgpr_build(self):
        self._ck(self.lib.bbmm_sgpr_build(self.h))

    def bbmm_sgpr_root_rows(self, row0: int, nrows: int):
        m = int(self._prob.Uind.shape[0])
        out = self._empty(nrows, m)
        self._ck(self.lib.bbmm_sgpr_root_rows(self.h, row0, nrows, _dptr(out)))
        return out

    def bbmm_kernel_mm(self, mode: int, M):
        n = self._shape[0]
        _check_dev(M, (n, M.shape[1]), "M")
        V = self._empty(n, M.shape[1])
        self._ck(self.lib.bbmm_kernel_mm(self.h, mode, _dptr(M), M.shape[1], _dptr(V)))
        return V

    def bbmm_pivoted_cholesky(self):
        n, _, _, k, _, _ = self._shape
        L = self.torch.empty(n, max(k, 1), dtype=self.torch.float64, device=self.device)
        piv = np.full(max(k, 1), -1, dtype=np.int64)
        rank = C.c_int64(0)
        self._ck(self.lib.bbmm_pivoted_cholesky(self.h, _dptr(L) if k > 0 else None,
                                                piv.ctypes.data_as(C.POINTER(C.c_int64)),
                                                C.byref(rank)))
        return L[:, :k], piv[:k], int(rank.value)

    def bbmm_precond_setup(self) -> float:
        out = C.c_double(0.0)
        self._ck(self.lib.bbmm_precond_setup(self.h, C.byref(out)))
        return float(out.value)

    def bbmm_precond_solve(self, R):
        n = self._shape[0]
        _check_dev(R, (n, R.shape[1]), "R")
        Z = self._empty(n, R.shape[1])
        self._ck(self.lib.bbmm_precond_solve(self.h, _dptr(R), R.shape[1], _dptr(Z)))
        return Z

    def bbmm_make_probes(self):
        n, _, t, _, _, _ = self._shape
        B = self._empty(n, t + 1)
        self._ck(self.lib.bbmm_make_probes(self.h, _dptr(B)))
        return B

    def bbmm_mbcg(self, mode: int, B):
        n, _, _, _, it, _ = self._shape
        c = B.shape[1]
        _check_dev(B, (n, c), "B")
        U = self._empty(n, c)
        alpha, beta, resid = (np.zeros((it, c)) for _ in range(3))
        iters = C.c_int64(0)
        self._ck(self.lib.bbmm_mbcg(self.h, mode, _dptr(B), c, _dptr(U), _dbl(alpha), _dbl(beta),
                                    _dbl(resid), C.byref(iters)))
        return U, alpha, beta, resid, int(iters.value)

    def bbmm_tridiag_eig_batched(self, diag: np.ndarray, off: np.ndarray, _fn=None):
        diag = np.ascontiguousarray(diag, dtype=np.float64)
        batch, m = diag.shape
        off = np.ascontiguousarray(off, dtype=np.float64).reshape(batch, max(m - 1, 0))
        vals, first = np.zeros((batch, m)), np.zeros((batch, m))
        offp = _dbl(off) if m > 1 else None
        fn = _fn if _fn is not None else self.lib.bbmm_tridiag_eig_batched
        self._ck(fn(self.h, _dbl(diag), offp, m, batch, _dbl(vals), _dbl(first)))
        return vals, first

    def bbmm_tridiag_eig_batched_noalloc(self, diag: np.ndarray, off: np.ndarray):
        return self.bbmm_tridiag_eig_batched(diag, off, _fn=self.lib.bbmm_tridiag_eig_batched_noalloc)

    def bbmm_slq_logdet(self):
        t = self._shape[2]
        out = C.c_double(0.0)
        terms = np.zeros(max(t, 1))
        self._ck(self.lib.bbmm_slq_logdet(self.h, C.byref(out), _dbl(terms)))
        return float(out.value), terms[:t]

    def bbmm_slq_from_coeffs(self, alpha: np.ndarray, beta: np.ndarray, rho0: np.ndarray, m_valid=None,
                             logdet_precond: float = 0.0):
        """alpha, beta: (p, t) coefficients of the probe columns; rho0: (t,); m_valid: (t,) or None."""
        alpha = np.ascontiguousarray(alpha, dtype=np.float64)
        beta = np.ascontiguousarray(beta, dtype=np.float64)
        rho0 = np.ascontiguousarray(rho0, dtype=np.float64)
        p, t = alpha.shape
        if beta.shape != (p, t) or rho0.shape != (t,):
            raise ValueError("alpha and beta must be (p, t), rho0 (t,)")
        mv = None
        mvp = None
        if m_valid is not None:
            mv = np.ascontiguousarray(m_valid, dtype=np.int64)
            if mv.shape != (t,):
                raise ValueError("m_valid must have t entries")
            mvp = mv.ctypes.data_as(C.POINTER(C.c_int64))
        out = C.c_double(0.0)
        terms = np.zeros(t)
        self._ck(self.lib.bbmm_slq_from_coeffs(self.h, _dbl(alpha), _dbl(beta), _dbl(rho0), mvp, p, t,
                                               float(logdet_precond), C.byref(out), _dbl(terms)))
        return float(out.value), terms

    def bbmm_dk_traces(self, U, W):
        n, _, t, _, _, nl = self._shape
        _check_dev(U, (n, t + 1), "U")
        _check_dev(W, (n, t), "W")
        trace, quad = np.zeros(nl + 2), np.zeros(nl + 2)
        self._ck(self.lib.bbmm_dk_traces(self.h, _dptr(U), _dptr(W), _dbl(trace), _dbl(quad)))
        return trace, quad

    def bbmm_predict_mean(self, Xstar, u0):
        n, d = self._shape[0], self._shape[1]
        ns = Xstar.shape[0]
        _check_dev(Xstar, (ns, d), "Xstar")
        _check_dev(u0, (n,), "u0")
        mean = self._empty(ns)
        self._ck(self.lib.bbmm_predict_mean(self.h, _dptr(Xstar), ns, _dptr(u0), _dptr(mean)))
        return mean

    def bbmm_predict_var(self, mode: int, Xstar):
        d = self._shape[1]
        ns = Xstar.shape[0]
        _check_dev(Xstar, (ns, d), "Xstar")
        var = self._empty(ns)
        iters, resid = C.c_int64(0), C.c_double(0.0)
        self._ck(self.lib.bbmm_predict_var(self.h, mode, _dptr(Xstar), ns, _dptr(var), C.byref(iters),
                                           C.byref(resid)))
        return var, int(iters.value), float(resid.value)


    # ---- attention --------------------------------------------------------------------------
    def _ordered(self, tensors, call):
        """Runs `call` (which allocates its outputs and queues work) with the context's stream current.  Where that is not
        the caller's stream, the work waits for what the caller has queued, the caller's stream waits for the work, and
        no tensor's memory is reused before both are done.  Refuses inputs whose gradients torch is to record: the result has no graph."""
        torch = self.torch
        if torch.is_grad_enabled():
            for t in tensors:
                if t.requires_grad:
                    raise ValueError("an input requires grad, but the call records no graph of gradients: make it under torch.no_grad(), "
                                     "or in the forward and backward of a torch.autograd.Function (bbmm_attend_grad, bbmm_bucket_bias_grad)")
        if torch._C._cuda_getCurrentRawStream(self.device.index) == self._raw_stream:
            return call()
        here = torch.cuda.current_stream(self.device)
        self._stream.wait_stream(here)
        with torch.cuda.stream(self._stream):
            out = call()
        for t in tensors:
            t.record_stream(self._stream)
        for t in out if isinstance(out, tuple) else (out,):
            if t is not None:
                t.record_stream(here)
        here.wait_stream(self._stream)
        return out

    def _work(self, nbytes: int):
        """(tensor to keep, pointer, size) of a workspace from torch's allocator on the current stream."""
        if nbytes == 0:
            return None, None, 0
        w = self.torch.empty(nbytes, dtype=self.torch.uint8, device=self.device)
        return w, w.data_ptr(), nbytes

    def _attend_bytes(self, a: _Attention, grad: bool) -> int:
        n = C.c_int64(0)
        self._ck(self.lib.bbmm_attend_workspace(self.h, C.byref(a), int(grad), C.byref(n)))
        return n.value

    def bbmm_attend_workspace(self, att: Attention, grad: bool = False) -> int:
        """Bytes that bbmm_attend (bbmm_attend_grad) takes from torch's allocator besides its outputs."""
        return self._attend_bytes(att.to_c(self.device), grad)

    def bbmm_attend(self, att: Attention):
        """(O, lse): (batch, nq, heads, dv) of Q's type and (batch, heads, nq) float32."""
        a = att.to_c(self.device)

        def call():
            b, h, nq = a.batch, a.heads, a.nq
            O = self.torch.empty((b, nq, h, a.dv), dtype=att.Q.dtype, device=self.device)
            lse = self.torch.empty((b, h, nq), dtype=self.torch.float32, device=self.device)
            w, wp, n = self._work(self._attend_bytes(a, False))
            self._ck(self.lib.bbmm_attend(self.h, C.byref(a), O.data_ptr(), lse.data_ptr(), wp, n))
            return O, lse

        return self._ordered(att.tensors(), call)

    def bbmm_attend_grad(self, att: Attention, O, lse, dO):
        """(dQ, dK, dV, dtable) of sum(dO * O); dtable is None without a table.  O, lse: from bbmm_attend of the same call."""
        a = att.to_c(self.device)
        t = att.Q.dtype
        shape = (a.batch, a.nq, a.heads, a.dv)
        _check_same(O, shape, t, self.device, "O")
        _check_same(lse, (a.batch, a.heads, a.nq), self.torch.float32, self.device, "lse")
        _check_same(dO, shape, t, self.device, "dO", dense=False)
        stride = (C.c_int64 * 3)(*dO.stride()[:3])

        def call():
            dQ, dK, dV = (self.torch.empty(x.shape, dtype=x.dtype, device=self.device) for x in (att.Q, att.K, att.V))
            dtable = None if att.table is None else self.torch.empty_like(att.table)
            w, wp, n = self._work(self._attend_bytes(a, True))
            self._ck(self.lib.bbmm_attend_grad(self.h, C.byref(a), O.data_ptr(), lse.data_ptr(), dO.data_ptr(), stride,
                                               dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(),
                                               None if dtable is None else dtable.data_ptr(), wp, n))
            return dQ, dK, dV, dtable

        return self._ordered(att.tensors() + [O, lse, dO], call)

    def bbmm_bucket_bias(self, table, edges, nq: int, nk: int, two_sided: bool = True, start: int = 0):
        """The bias as a matrix (heads, nq, nk) of the table's type: table[h, bucket(j - i - start)]."""
        kind, e = _type_of(table, "table"), _edges(edges)
        _check_same(table, (table.shape[0], (len(e) + 1) * (2 if two_sided else 1)), table.dtype, self.device, "table")

        def call():
            B = self.torch.empty(table.shape[0], nq, nk, dtype=table.dtype, device=self.device)
            self._ck(self.lib.bbmm_bucket_bias(self.h, kind, table.data_ptr(), table.shape[0], nq, nk, len(e), e,
                                               int(bool(two_sided)), _int64(start), B.data_ptr()))
            return B

        return self._ordered([table], call)

    def bbmm_bucket_bias_workspace(self, batch: int, heads: int, nq: int, nk: int, n_edges: int, two_sided: bool = True) -> int:
        """Bytes that bbmm_bucket_bias_grad takes from torch's allocator besides its output."""
        n = C.c_int64(0)
        self._ck(self.lib.bbmm_bucket_bias_workspace(self.h, batch, heads, nq, nk, n_edges, int(bool(two_sided)),
                                                     C.byref(n)))
        return n.value

    def bbmm_bucket_bias_grad(self, dB, edges, two_sided: bool = True, start: int = 0):
        """Gradient (heads, buckets) of the table from that of the matrix, dB (batch, heads, nq, nk), summed over the batch."""
        kind, e = _type_of(dB, "dB"), _edges(edges)
        if dB.dim() != 4:
            raise ValueError("dB must have four dimensions (batch, head, nq, nk)")
        _check_same(dB, dB.shape, dB.dtype, self.device, "dB")
        b, h, nq, nk = dB.shape

        def call():
            dtable = self.torch.empty(h, (len(e) + 1) * (2 if two_sided else 1), dtype=dB.dtype, device=self.device)
            w, wp, n = self._work(self.bbmm_bucket_bias_workspace(b, h, nq, nk, len(e), two_sided))
            self._ck(self.lib.bbmm_bucket_bias_grad(self.h, kind, dB.data_ptr(), b, h, nq, nk, len(e), e, int(bool(two_sided)),
                                                    _int64(start), dtable.data_ptr(), wp, n))
            return dtable

        return self._ordered([dB], call)


def problem_from_workload(w, mode: int, device="cuda:0") -> Problem:
    """Uploads a paper_1809_11165_amd.inputs.Workload (host arrays) and wraps it as a Problem."""
    import torch
    dev = torch.device(device)

    def up(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev)

    E1 = up(w.E1) if w.k > 0 else None
    Uind = up(w.Uind) if mode == MODE_SGPR else None
    return Problem(kernel=w.kernel, mode=mode, X=up(w.X), y=up(w.y), lengthscale=w.lengthscale,
                   outputscale=w.outputscale, noise=w.noise, E1=E1, E2=up(w.E2), k=w.k,
                   max_iters=w.iters, tol=w.tol, Uind=Uind, jitter_rel=w.jitter_rel)
