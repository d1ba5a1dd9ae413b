"""Thin ctypes binding of the C ABI in include/comet.h.

Argument marshalling only: every function checks dtypes / devices / contiguity of the torch
tensors it is given, passes their device pointers and the current HIP stream to the library,
and wraps what comes back.  PyTorch is used for device memory and streams; all arithmetic runs
in the HIP kernels of libcomet_hip.so.  There is no fallback: if the shared library is missing
the import of this module's functions fails with an error that says how to build it.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcomet_hip.so")

COMET_D, COMET_CU, COMET_CN, COMET_S = 0, 1, 2, 3
COMET_BORROW, COMET_COPY, COMET_VALIDATE, COMET_LEAN = 0, 1, 2, 4
COMET_OK = 0
COMET_MAX_ORDER = 4
COMET_F32, COMET_BF16, COMET_F16 = 0, 1, 2
COMET_BY_COORDINATE = 1
COMET_MAX_TOP, COMET_MAX_BEAMS, COMET_DISTILL_STAT = 1024, 256, 7

_STATUS_NAMES = {0: "COMET_OK", 1: "COMET_ERR_INVALID_ARG", 2: "COMET_ERR_BAD_FORMAT", 3: "COMET_ERR_SHAPE",
                 4: "COMET_ERR_UNSUPPORTED", 5: "COMET_ERR_ALLOC", 6: "COMET_ERR_DEVICE"}

EXPORTS = ["comet_tensor_create", "comet_tensor_destroy", "comet_tensor_info", "comet_spmv", "comet_spmm",
           "comet_ttv", "comet_ttm", "comet_mttkrp", "comet_status_string", "comet_tensor_set_variant",
           "comet_tensor_reorder", "comet_tensor_convert", "comet_tensor_reserve", "comet_spmv_static",
           "comet_calibrate_read", "comet_calibrate_gather", "comet_spmv_axpby", "comet_spmm_axpby",
           "comet_mttkrp_axpby", "comet_rows_topk_work", "comet_rows_topk", "comet_distill_work", "comet_distill_forward",
           "comet_distill_backward", "comet_distill_step", "comet_beam_select_work", "comet_beam_select", "comet_beam_reorder"]


class CometError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _lib().comet_status_string(status).decode() if _LIB is not None else ""
        super().__init__("%s: %s (%s)" % (where, _STATUS_NAMES.get(status, status), msg))


class _Info(ctypes.Structure):
    _fields_ = [("order", ctypes.c_int32),
                ("dims", ctypes.c_int64 * COMET_MAX_ORDER),
                ("levels", ctypes.c_int32 * COMET_MAX_ORDER),
                ("pos", ctypes.c_void_p * COMET_MAX_ORDER),
                ("pos_len", ctypes.c_int64 * COMET_MAX_ORDER),
                ("crd", ctypes.c_void_p * COMET_MAX_ORDER),
                ("crd_len", ctypes.c_int64 * COMET_MAX_ORDER),
                ("vals", ctypes.c_void_p),
                ("nvals", ctypes.c_int64),
                ("mode_of_level", ctypes.c_int32 * COMET_MAX_ORDER),
                ("heavy_rows", ctypes.c_int64),
                ("heavy_nnz", ctypes.c_int64),
                ("heavy_stream_bytes", ctypes.c_int64)]


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("%s is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
                              "or paper_2102_05187_amd.build.build())" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        lib.comet_tensor_create.argtypes = [ctypes.POINTER(vp), ci, vp, vp, vp, vp, vp, vp, vp, i64, ctypes.c_uint, vp]
        lib.comet_tensor_destroy.argtypes = [vp]
        lib.comet_tensor_info.argtypes = [vp, ctypes.POINTER(_Info)]
        lib.comet_spmv.argtypes = [vp, vp, vp, vp]
        lib.comet_spmv_static.argtypes = [vp, vp, vp, vp]
        lib.comet_tensor_reserve.argtypes = [vp, i64, vp]
        lib.comet_calibrate_read.argtypes = [vp, i64, vp, vp]
        lib.comet_calibrate_gather.argtypes = [vp, i64, i64, i64, vp, vp]
        lib.comet_spmm.argtypes = [vp, vp, i64, vp, vp]
        lib.comet_ttv.argtypes = [vp, ci, vp, ctypes.POINTER(vp), vp]
        lib.comet_ttm.argtypes = [vp, ci, vp, i64, ctypes.POINTER(vp), vp]
        lib.comet_mttkrp.argtypes = [vp, ci, vp, i64, vp, vp]
        f64 = ctypes.c_double
        lib.comet_spmv_axpby.argtypes = [vp, f64, vp, f64, vp, vp]
        lib.comet_spmm_axpby.argtypes = [vp, f64, vp, i64, f64, vp, vp]
        lib.comet_mttkrp_axpby.argtypes = [vp, ci, f64, vp, i64, f64, vp, vp]
        lib.comet_tensor_set_variant.argtypes = [vp, ci]
        lib.comet_tensor_reorder.argtypes = [vp, vp, ctypes.POINTER(vp), vp]
        lib.comet_tensor_convert.argtypes = [vp, vp, vp, ctypes.POINTER(vp), vp]
        pi64 = ctypes.POINTER(i64)
        lib.comet_rows_topk_work.argtypes = [ci, i64, i64, i64, pi64]
        lib.comet_rows_topk.argtypes = [vp, ci, i64, i64, i64, f64, i64, ctypes.c_uint, vp, vp, vp, vp, i64, vp]
        lib.comet_distill_work.argtypes = [ci, i64, i64, pi64]
        rows = [vp, ci, i64, i64, i64, vp, i64, vp, vp, vp, f64, vp]
        lib.comet_distill_forward.argtypes = rows + [vp, vp, vp, i64, vp]
        lib.comet_distill_backward.argtypes = rows + [vp, vp, vp, i64, vp]
        lib.comet_distill_step.argtypes = rows + [vp, vp, i64, vp, i64, vp]
        lib.comet_beam_select_work.argtypes = [ci, i64, i64, i64, i64, pi64]
        lib.comet_beam_select.argtypes = [vp, ci, i64, i64, i64, i64, vp, vp, ctypes.c_int32, i64, vp, vp, vp, vp, i64, vp]
        lib.comet_beam_reorder.argtypes = [vp, i64, i64, i64, i64, i64, i64, i64, i64, vp, vp]
        lib.comet_status_string.argtypes = [ci]
        lib.comet_status_string.restype = ctypes.c_char_p
        for n in EXPORTS:
            if n != "comet_status_string":
                getattr(lib, n).restype = ci
        _LIB = lib
    return _LIB


def _check(status: int, where: str):
    if status != COMET_OK:
        raise CometError(status, where)


# The current stream's address without a Stream object around it, which takes 2.8 us to make: 4096 rows x 10 nonzeros, one call
# among others, SpMV 7.7 -> 4.8 us, SpMM with 32 columns 8.3 -> 5.5.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _dev(t: Optional[torch.Tensor], dtype, what: str) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor in device memory" % what)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (what, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None or t.numel() == 0 else t.data_ptr()


class _DeviceView:
    """Exposes a raw device pointer through __cuda_array_interface__ so torch can wrap it."""

    def __init__(self, ptr: int, n: int, typestr: str, owner):
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": typestr, "data": (ptr, False), "version": 2}
        self._owner = owner


class Tensor:
    """A library tensor handle plus the torch tensors it borrows (kept alive with it)."""

    def __init__(self, handle: int, keep: Sequence = (), parent: "Tensor" = None):
        self._h = ctypes.c_void_p(handle)
        self._keep = list(keep)
        self._parent = parent      # a result shares level arrays with its input
        self._dims = None
        self._mode_dims = None

    @property
    def handle(self) -> ctypes.c_void_p:
        if not self._h:
            raise ValueError("tensor handle was destroyed")
        return self._h

    def info(self) -> _Info:
        inf = _Info()
        _check(_lib().comet_tensor_info(self.handle, ctypes.byref(inf)), "comet_tensor_info")
        return inf

    def _wrap(self, ptr, n, typestr, dtype, copy=True):
        if not ptr or n == 0:
            return torch.empty(0, dtype=dtype, device="cuda")
        view = torch.as_tensor(_DeviceView(ptr, n, typestr, self), device="cuda")
        return view.clone() if copy else view

    def levels(self) -> List[int]:
        inf = self.info()
        return [int(inf.levels[l]) for l in range(inf.order)]

    def dims(self) -> List[int]:
        # sizes never change for a handle: looked up once (the products are launch-bound on small inputs)
        if self._dims is None:
            inf = self.info()
            self._dims = [int(inf.dims[l]) for l in range(inf.order)]
        return list(self._dims)

    def mode_of_level(self) -> List[int]:
        inf = self.info()
        return [int(inf.mode_of_level[l]) for l in range(inf.order)]

    def heavy_plan(self):
        """(rows, nonzeros) that comet_spmm hands to its heavy-row sweep; (0, 0) when none is planned."""
        inf = self.info()
        return int(inf.heavy_rows), int(inf.heavy_nnz)

    def heavy_stream_bytes(self) -> int:
        """Device memory held by the re-ordered copy of the heavy rows that the sweep reads (0: no sweep planned)."""
        return int(self.info().heavy_stream_bytes)

    def mode_dims(self) -> List[int]:
        """Sizes indexed by tensor mode (dims() is indexed by level)."""
        if self._mode_dims is None:
            inf = self.info()
            out = [0] * inf.order
            for l in range(inf.order):
                out[int(inf.mode_of_level[l])] = int(inf.dims[l])
            self._mode_dims = out
        return list(self._mode_dims)

    def pos(self, l: int) -> Optional[torch.Tensor]:
        inf = self.info()
        return None if inf.pos_len[l] == 0 else self._wrap(inf.pos[l], inf.pos_len[l], "<i4", torch.int32)

    def crd(self, l: int) -> Optional[torch.Tensor]:
        inf = self.info()
        if int(inf.levels[l]) == COMET_D:
            return None
        return self._wrap(inf.crd[l], inf.crd_len[l], "<i4", torch.int32)

    def vals(self, copy: bool = True) -> torch.Tensor:
        """The value array; copy=False returns a view of the library's memory (valid while the handle lives)."""
        inf = self.info()
        return self._wrap(inf.vals, inf.nvals, "<f8", torch.float64, copy)

    def reserve(self, R: int, stream=None) -> "Tensor":
        _check(_lib().comet_tensor_reserve(self.handle, int(R), _stream(stream)), "comet_tensor_reserve")
        return self

    def set_variant(self, variant: int) -> "Tensor":
        _check(_lib().comet_tensor_set_variant(self.handle, variant), "comet_tensor_set_variant")
        return self

    def destroy(self):
        if self._h:
            _check(_lib().comet_tensor_destroy(self._h), "comet_tensor_destroy")
            self._h = ctypes.c_void_p(None)
            self._keep = []

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def comet_tensor_create(dims: Sequence[int], levels: Sequence[int], pos: Sequence[Optional[torch.Tensor]],
                        crd: Sequence[Optional[torch.Tensor]], vals: torch.Tensor,
                        flags: int = COMET_VALIDATE, stream=None) -> Tensor:
    order = len(dims)
    if not (len(levels) == len(pos) == len(crd) == order):
        raise ValueError("dims, levels, pos and crd must have one entry per level")
    pos = [_dev(p, torch.int32, "pos[%d]" % l) for l, p in enumerate(pos)]
    crd = [_dev(c, torch.int32, "crd[%d]" % l) for l, c in enumerate(crd)]
    vals = _dev(vals, torch.float64, "vals")
    c_dims = (ctypes.c_int64 * order)(*[int(d) for d in dims])
    c_lv = (ctypes.c_int * order)(*[int(t) for t in levels])
    c_pos = (ctypes.c_void_p * order)(*[_ptr(p) for p in pos])
    c_crd = (ctypes.c_void_p * order)(*[_ptr(c) for c in crd])
    c_pl = (ctypes.c_int64 * order)(*[0 if p is None else p.numel() for p in pos])
    c_cl = (ctypes.c_int64 * order)(*[0 if c is None else c.numel() for c in crd])
    out = ctypes.c_void_p(None)
    st = _lib().comet_tensor_create(ctypes.byref(out), order, c_dims, c_lv, c_pos, c_pl, c_crd, c_cl,
                                    _ptr(vals), vals.numel(), flags, _stream(stream))
    _check(st, "comet_tensor_create")
    keep = [] if (flags & COMET_COPY) else [*pos, *crd, vals]
    return Tensor(out.value, keep)


def comet_tensor_destroy(t: Tensor):
    t.destroy()


def comet_tensor_reorder(X: Tensor, mode_order: Sequence[int], stream=None) -> Tensor:
    order = len(X.dims())
    if len(mode_order) != order:
        raise CometError(1, "comet_tensor_reorder")
    c_order = (ctypes.c_int32 * order)(*[int(m) for m in mode_order])
    out = ctypes.c_void_p(None)
    _check(_lib().comet_tensor_reorder(X.handle, c_order, ctypes.byref(out), _stream(stream)), "comet_tensor_reorder")
    return Tensor(out.value)


def comet_tensor_convert(X: Tensor, mode_order: Sequence[int], levels: Sequence[int], stream=None) -> Tensor:
    order = len(X.dims())
    if len(mode_order) != order or len(levels) != order:
        raise CometError(1, "comet_tensor_convert")
    c_order = (ctypes.c_int32 * order)(*[int(m) for m in mode_order])
    c_lv = (ctypes.c_int * order)(*[int(t) for t in levels])
    out = ctypes.c_void_p(None)
    _check(_lib().comet_tensor_convert(X.handle, c_order, c_lv, ctypes.byref(out), _stream(stream)), "comet_tensor_convert")
    return Tensor(out.value)


def comet_spmv(A: Tensor, x: torch.Tensor, y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    x = _dev(x, torch.float64, "x")
    dims = A.dims()
    if len(dims) != 2:
        raise CometError(4, "comet_spmv")
    I, J = dims
    if x.numel() != J:
        raise CometError(3, "comet_spmv")
    if y is None:
        y = torch.empty(I, dtype=torch.float64, device=x.device)
    y = _dev(y, torch.float64, "y")
    if y.numel() != I:
        raise CometError(3, "comet_spmv")
    _check(_lib().comet_spmv(A.handle, x.data_ptr(), y.data_ptr(), _stream(stream)), "comet_spmv")
    return y


def comet_spmv_axpby(A: Tensor, alpha: float, x: torch.Tensor, beta: float, y: torch.Tensor, stream=None) -> torch.Tensor:
    """y = alpha * A x + beta * y, in place."""
    x, y = _dev(x, torch.float64, "x"), _dev(y, torch.float64, "y")
    if len(A.dims()) != 2:
        raise CometError(4, "comet_spmv_axpby")
    I, J = A.dims()
    if x.numel() != J or y.numel() != I:
        raise CometError(3, "comet_spmv_axpby")
    _check(_lib().comet_spmv_axpby(A.handle, float(alpha), x.data_ptr(), float(beta), y.data_ptr(), _stream(stream)),
           "comet_spmv_axpby")
    return y


def comet_spmm_axpby(A: Tensor, alpha: float, B: torch.Tensor, beta: float, C: torch.Tensor, stream=None) -> torch.Tensor:
    """C = alpha * A B + beta * C, in place."""
    B, C = _dev(B, torch.float64, "B"), _dev(C, torch.float64, "C")
    if len(A.dims()) != 2:
        raise CometError(4, "comet_spmm_axpby")
    I, J = A.dims()
    if B.dim() != 2 or B.shape[0] != J or tuple(C.shape) != (I, B.shape[1]):
        raise CometError(3, "comet_spmm_axpby")
    _check(_lib().comet_spmm_axpby(A.handle, float(alpha), B.data_ptr(), B.shape[1], float(beta), C.data_ptr(),
                                   _stream(stream)), "comet_spmm_axpby")
    return C


def comet_spmv_static(A: Tensor, x: torch.Tensor, y: torch.Tensor, stream=None) -> torch.Tensor:
    """comet_spmv for callers that cannot allocate: the caller passes y, the library's scratch is static."""
    x, y = _dev(x, torch.float64, "x"), _dev(y, torch.float64, "y")
    if len(A.dims()) != 2:
        raise CometError(4, "comet_spmv_static")
    I, J = A.dims()
    if x.numel() != J or y.numel() != I:
        raise CometError(3, "comet_spmv_static")
    _check(_lib().comet_spmv_static(A.handle, x.data_ptr(), y.data_ptr(), _stream(stream)), "comet_spmv_static")
    return y


def comet_calibrate_read(data: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    data, sink = _dev(data, torch.float64, "data"), _dev(sink, torch.float64, "sink")
    _check(_lib().comet_calibrate_read(data.data_ptr(), data.numel(), sink.data_ptr(), _stream(stream)), "comet_calibrate_read")


def comet_calibrate_gather(table: torch.Tensor, gathers: int, sink: torch.Tensor, stream=None) -> None:
    table, sink = _dev(table, torch.float64, "table"), _dev(sink, torch.float64, "sink")
    if table.dim() != 2:
        raise CometError(3, "comet_calibrate_gather")
    _check(_lib().comet_calibrate_gather(table.data_ptr(), table.shape[0], table.shape[1], int(gathers), sink.data_ptr(),
                                         _stream(stream)), "comet_calibrate_gather")


def comet_spmm(A: Tensor, B: torch.Tensor, C: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    B = _dev(B, torch.float64, "B")
    dims = A.dims()
    if len(dims) != 2:
        raise CometError(4, "comet_spmm")
    I, J = dims
    if B.dim() != 2 or B.shape[0] != J:
        raise CometError(3, "comet_spmm")
    R = B.shape[1]
    if C is None:
        C = torch.empty((I, R), dtype=torch.float64, device=B.device)
    C = _dev(C, torch.float64, "C")
    if tuple(C.shape) != (I, R):
        raise CometError(3, "comet_spmm")
    _check(_lib().comet_spmm(A.handle, B.data_ptr(), R, C.data_ptr(), _stream(stream)), "comet_spmm")
    return C


def comet_ttv(X: Tensor, mode: int, v: torch.Tensor, Y: Optional[Tensor] = None, stream=None) -> Tensor:
    v = _dev(v, torch.float64, "v")
    dims = X.mode_dims()
    if len(dims) != 3:
        raise CometError(4, "comet_ttv")
    if 0 <= mode < 3 and v.numel() != dims[mode]:
        raise CometError(3, "comet_ttv")
    h = ctypes.c_void_p(Y.handle.value if Y is not None else None)
    _check(_lib().comet_ttv(X.handle, mode, v.data_ptr(), ctypes.byref(h), _stream(stream)), "comet_ttv")
    return Y if Y is not None else Tensor(h.value, parent=X)


def comet_ttm(X: Tensor, mode: int, U: torch.Tensor, Y: Optional[Tensor] = None, stream=None) -> Tensor:
    U = _dev(U, torch.float64, "U")
    dims = X.mode_dims()
    if len(dims) != 3:
        raise CometError(4, "comet_ttm")
    if U.dim() != 2 or (0 <= mode < 3 and U.shape[0] != dims[mode]):
        raise CometError(3, "comet_ttm")
    h = ctypes.c_void_p(Y.handle.value if Y is not None else None)
    _check(_lib().comet_ttm(X.handle, mode, U.data_ptr(), U.shape[1], ctypes.byref(h), _stream(stream)), "comet_ttm")
    return Y if Y is not None else Tensor(h.value, parent=X)


def comet_mttkrp(X: Tensor, mode: int, factors: Sequence[Optional[torch.Tensor]],
                 M: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    dims = X.mode_dims()
    if len(dims) != 3 or len(factors) != 3:
        raise CometError(4, "comet_mttkrp")
    fs = [None if (f is None or l == mode) else _dev(f, torch.float64, "factors[%d]" % l) for l, f in enumerate(factors)]
    R = None
    for l, f in enumerate(fs):
        if f is None:
            continue
        if f.dim() != 2 or f.shape[0] != dims[l] or (R is not None and f.shape[1] != R):
            raise CometError(3, "comet_mttkrp")
        R = f.shape[1]
    if R is None or not (0 <= mode < 3):
        raise CometError(1, "comet_mttkrp")
    dev = next(f for f in fs if f is not None).device
    if M is None:
        M = torch.empty((dims[mode], R), dtype=torch.float64, device=dev)
    M = _dev(M, torch.float64, "M")
    if tuple(M.shape) != (dims[mode], R):
        raise CometError(3, "comet_mttkrp")
    c_f = (ctypes.c_void_p * 3)(*[_ptr(f) for f in fs])
    _check(_lib().comet_mttkrp(X.handle, mode, c_f, R, M.data_ptr(), _stream(stream)), "comet_mttkrp")
    return M


def comet_mttkrp_axpby(X: Tensor, mode: int, alpha: float, factors: Sequence[Optional[torch.Tensor]], beta: float,
                       M: torch.Tensor, stream=None) -> torch.Tensor:
    """M = alpha * MTTKRP(X, factors) + beta * M, in place."""
    dims = X.mode_dims()
    if len(dims) != 3 or len(factors) != 3:
        raise CometError(4, "comet_mttkrp_axpby")
    fs = [None if (f is None or l == mode) else _dev(f, torch.float64, "factors[%d]" % l) for l, f in enumerate(factors)]
    R = None
    for l, f in enumerate(fs):
        if f is None:
            continue
        if f.dim() != 2 or f.shape[0] != dims[l] or (R is not None and f.shape[1] != R):
            raise CometError(3, "comet_mttkrp_axpby")
        R = f.shape[1]
    if R is None or not (0 <= mode < 3):
        raise CometError(1, "comet_mttkrp_axpby")
    M = _dev(M, torch.float64, "M")
    if tuple(M.shape) != (dims[mode], R):
        raise CometError(3, "comet_mttkrp_axpby")
    c_f = (ctypes.c_void_p * 3)(*[_ptr(f) for f in fs])
    _check(_lib().comet_mttkrp_axpby(X.handle, mode, float(alpha), c_f, R, float(beta), M.data_ptr(), _stream(stream)),
           "comet_mttkrp_axpby")
    return M


def from_levels(T, flags: int = COMET_VALIDATE, stream=None) -> Tensor:
    """Create a handle from a synth.LevelTensor-like object (dims, tags, pos, crd, vals on the GPU)."""
    return comet_tensor_create(T.dims, T.tags, T.pos, T.crd, T.vals, flags, stream)


# ---- dense rows over a vocabulary and their sparse top part -------------------------------------------------------------
_TYPES = {torch.float32: COMET_F32, torch.bfloat16: COMET_BF16, torch.float16: COMET_F16}


def _rows(Z: torch.Tensor, what: str = "Z"):
    """(pointer, type, rows, columns, distance of rows) of a matrix whose rows may lie apart but not its columns."""
    if not isinstance(Z, torch.Tensor) or not Z.is_cuda:
        raise TypeError("%s must be a torch tensor in device memory" % what)
    if Z.dtype not in _TYPES:
        raise TypeError("%s must have dtype float32, bfloat16 or float16, got %s" % (what, Z.dtype))
    if Z.dim() != 2:
        raise ValueError("%s must have two dimensions" % what)
    (N, V), (ld, step) = Z.shape, Z.stride()
    if (step != 1 and V > 1) or (ld < V and N > 1):
        raise ValueError("%s must have its columns next to each other and rows that do not overlap" % what)
    return Z.data_ptr(), _TYPES[Z.dtype], N, V, ld if N > 1 else V


def _given(t: Optional[torch.Tensor], dtype, shape, what: str, device) -> Optional[torch.Tensor]:
    """An operand of a stated shape on the same device as the others."""
    # all at once where nothing is wrong: the smallest calls take 7 us on the device, and each check done alone 0.1
    if t is None or (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous()):
        return t
    _dev(t, dtype, what)
    if tuple(t.shape) != shape:
        raise ValueError("%s must have shape %s, got %s" % (what, shape, tuple(t.shape)))
    if t.device != device:
        raise ValueError("%s must be on %s" % (what, device))
    return t


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Memory for a call on `stream`, from that stream's pool: what the current stream's pool has free may still be in use by work that
    the current stream has before it."""
    with torch.cuda.stream(stream):
        return torch.empty(*shape, dtype=dtype, device=device)


def _new(t: Optional[torch.Tensor], dtype, shape, what: str, device, stream) -> torch.Tensor:
    """A result: the caller's tensor, which is marked as changed (automatic differentiation then refuses to use what it kept of it), or a
    new one, which the current stream is expected to go on with."""
    if t is not None:
        _given(t, dtype, shape, what, device)
        torch.autograd.graph.increment_version(t)
        return t
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)
    t = _empty(shape, dtype, device, stream)
    t.record_stream(torch.cuda.current_stream(device))
    return t


@functools.lru_cache(maxsize=1024)
def _work_bytes(call: str, *sizes) -> int:
    need = ctypes.c_int64(0)
    _check(getattr(_lib(), call + "_work")(*sizes, ctypes.byref(need)), call)
    return need.value


def _work(need: int, device, stream):
    """(tensor, pointer) of scratch for one call: its memory goes back to the pool of the stream that the call runs on."""
    if need == 0:
        return None, None
    t = torch.empty(need, dtype=torch.uint8, device=device) if stream is None else _empty((need,), torch.uint8, device, stream)
    return t, t.data_ptr()


def _call(name: str, device, stream, *args) -> None:
    """One of the calls on dense rows, on its operands' device, with the stream (that device's current one: None) as the last argument."""
    call = getattr(_lib(), name)
    if stream is not None and stream.device != device:
        raise ValueError("stream must be one of %s, where the operands are" % device)
    if stream is None and _raw_stream is not None and _raw_device is not None and _raw_device() == device.index:
        status = call(*args, _raw_stream(device.index))
    else:
        with torch.cuda.device(device):
            status = call(*args, _stream(stream))
    if status != COMET_OK:
        raise CometError(status, name)


def comet_rows_topk(Z: torch.Tensor, K: int, scale: float = 1.0, by_coordinate: bool = False, crd: Optional[torch.Tensor] = None,
                    vals: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stream=None):
    """(crd, vals, lse): the K largest elements of every row of Z and log sum exp(scale * row)."""
    ptr, kind, N, V, ld = _rows(Z)
    K, dev = int(K), Z.device
    need = _work_bytes("comet_rows_topk", kind, N, V, K)
    crd = _new(crd, torch.int32, (N, K), "crd", dev, stream)
    vals = _new(vals, torch.float32, (N, K), "vals", dev, stream)
    lse = _new(lse, torch.float32, (N,), "lse", dev, stream)
    work, wptr = _work(need, dev, stream)
    _call("comet_rows_topk", dev, stream, ptr, kind, N, V, ld, float(scale), K, COMET_BY_COORDINATE if by_coordinate else 0, crd.data_ptr(),
          vals.data_ptr(), lse.data_ptr(), wptr, need)
    return crd, vals, lse


def _teacher(Z, crd, tvals, pos, tlse, scale, weight):
    """The arguments that the three distillation calls share."""
    ptr, kind, N, V, ld = _rows(Z)
    dev, of_rows = Z.device, (N,)
    if not isinstance(crd, torch.Tensor) or crd.dim() != (2 if pos is None else 1):
        raise ValueError("crd must be an [N, K] matrix where there is no pos, and have one dimension where there is one")
    shape, K = crd.shape, 0
    if pos is None:
        K = shape[1]
        shape = (N, K)
    else:
        _given(pos, torch.int32, (N + 1,), "pos", dev)
    _given(crd, torch.int32, tuple(shape), "crd", dev)
    _given(tvals, torch.float32, tuple(shape), "tvals", dev)
    if tvals is None:
        raise ValueError("tvals are missing")
    _given(tlse, torch.float32, of_rows, "tlse", dev)
    _given(weight, torch.float32, of_rows, "weight", dev)
    return N, V, kind, dev, (ptr, kind, N, V, ld, None if pos is None else pos.data_ptr(), K, crd.data_ptr(), tvals.data_ptr(),
                             None if tlse is None else tlse.data_ptr(), float(scale), None if weight is None else weight.data_ptr())


def comet_distill_forward(Z: torch.Tensor, crd: torch.Tensor, tvals: torch.Tensor, pos: Optional[torch.Tensor] = None,
                          tlse: Optional[torch.Tensor] = None, scale: float = 1.0, weight: Optional[torch.Tensor] = None,
                          loss: Optional[torch.Tensor] = None, stat: Optional[torch.Tensor] = None, stream=None):
    """(loss, stat): the loss of every row, and what comet_distill_backward needs of it.  Neither is part of an autograd graph."""
    N, V, kind, dev, args = _teacher(Z, crd, tvals, pos, tlse, scale, weight)
    need = _work_bytes("comet_distill", kind, N, V)
    loss = _new(loss, torch.float32, (N,), "loss", dev, stream)
    stat = _new(stat, torch.float64, (N, COMET_DISTILL_STAT), "stat", dev, stream)
    work, wptr = _work(need, dev, stream)
    _call("comet_distill_forward", dev, stream, *args, loss.data_ptr(), stat.data_ptr(), wptr, need)
    return loss, stat


def _gradient(Z, dZ, stream):
    if dZ is None:
        dZ = _new(None, Z.dtype, Z.shape, "dZ", Z.device, stream)
        return dZ, dZ.data_ptr(), Z.shape[1]
    if dZ.dtype != Z.dtype or dZ.shape != Z.shape or dZ.device != Z.device:
        raise ValueError("dZ must have Z's shape, dtype and device")
    ptr, _, _, _, ld = _rows(dZ, "dZ")
    torch.autograd.graph.increment_version(dZ)
    return dZ, ptr, ld


def comet_distill_backward(Z: torch.Tensor, crd: torch.Tensor, tvals: torch.Tensor, stat: torch.Tensor, pos: Optional[torch.Tensor] = None,
                           tlse: Optional[torch.Tensor] = None, scale: float = 1.0, weight: Optional[torch.Tensor] = None,
                           dloss: Optional[torch.Tensor] = None, dZ: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dZ, which may be Z itself: the gradient of sum(dloss * loss) by Z, from the stat of the forward call with the same arguments."""
    N, V, kind, dev, args = _teacher(Z, crd, tvals, pos, tlse, scale, weight)
    _given(stat, torch.float64, (N, COMET_DISTILL_STAT), "stat", dev)
    _given(dloss, torch.float32, (N,), "dloss", dev)
    dZ, out, ldo = _gradient(Z, dZ, stream)
    _call("comet_distill_backward", dev, stream, *args, _ptr(stat), _ptr(dloss), out, ldo)
    return dZ


def comet_distill_step(Z: torch.Tensor, crd: torch.Tensor, tvals: torch.Tensor, pos: Optional[torch.Tensor] = None,
                       tlse: Optional[torch.Tensor] = None, scale: float = 1.0, weight: Optional[torch.Tensor] = None,
                       loss: Optional[torch.Tensor] = None, dZ: Optional[torch.Tensor] = None, stream=None):
    """(loss, dZ): both at once, for a training step that knows its rows' weights; dZ may be Z itself."""
    N, V, kind, dev, args = _teacher(Z, crd, tvals, pos, tlse, scale, weight)
    need = _work_bytes("comet_distill", kind, N, V)
    loss = _new(loss, torch.float32, (N,), "loss", dev, stream)
    dZ, out, ldo = _gradient(Z, dZ, stream)
    work, wptr = _work(need, dev, stream)
    _call("comet_distill_step", dev, stream, *args, loss.data_ptr(), out, ldo, wptr, need)
    return loss, dZ


def comet_beam_select(Z: torch.Tensor, score: torch.Tensor, n: int, finished: Optional[torch.Tensor] = None, eos: int = 0, stream=None):
    """(score, parent, token), each [B, n]: the best continuations of every batch's beams.  Z: [B, W, V] logits."""
    if not isinstance(Z, torch.Tensor) or Z.dim() != 3:
        raise ValueError("Z must have three dimensions")
    B, W, V = Z.shape
    if B > 1 and W > 1 and Z.stride(0) != W * Z.stride(1):
        raise ValueError("Z must have its batches' rows at one distance")
    ptr, kind, _, _, ld = _rows(Z.flatten(0, 1))
    n, dev = int(n), Z.device
    _given(score, torch.float32, (B, W), "score", dev)
    if finished is not None:
        if isinstance(finished, torch.Tensor) and finished.dtype == torch.bool:
            finished = finished.view(torch.uint8)
        _given(finished, torch.uint8, (B, W), "finished", dev)
    need = _work_bytes("comet_beam_select", kind, B, W, V, n)
    best = _new(None, torch.float32, (B, n), "score", dev, stream)
    parent = _new(None, torch.int32, (B, n), "parent", dev, stream)
    token = _new(None, torch.int32, (B, n), "token", dev, stream)
    work, wptr = _work(need, dev, stream)
    _call("comet_beam_select", dev, stream, ptr, kind, B, W, V, ld, score.data_ptr(), _ptr(finished), int(eos), n, best.data_ptr(), parent.data_ptr(),
          token.data_ptr(), wptr, need)
    return best, parent, token


@functools.lru_cache(maxsize=256)
def _pieces(shape, strides, size):
    """The layout of [B, W, ...] states in bytes: strides of batch and beam, and what a beam holds as equal pieces (number, distance, length).
    A beam's dimensions are taken in the order of their memory: all of them move alike."""
    dims = sorted(((n, s) for n, s in zip(shape[2:], strides[2:]) if n != 1), key=lambda d: -d[1])
    inner = 1
    while dims and dims[-1][1] == inner:
        inner *= dims.pop()[0]
    outer, stride = dims.pop() if dims else (1, 0)
    while dims and dims[-1][1] == outer * stride:
        outer *= dims.pop()[0]
    if dims:
        raise ValueError("a state's beam must be pieces of one length at one distance")
    return strides[0] * size, strides[1] * size, outer, stride * size, inner * size


def comet_beam_reorder(states: Sequence[torch.Tensor], parent: torch.Tensor, stream=None) -> None:
    """states[i][b, w] = old states[i][b, parent[b, w]], in place; the states are [B, W, ...] tensors, of one layout or several."""
    if not isinstance(parent, torch.Tensor) or parent.dim() != 2:
        raise ValueError("parent must have two dimensions")
    B, W = parent.shape
    _dev(parent, torch.int32, "parent")
    states, groups, kind = list(states), {}, None
    for t in states:
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError("states must be torch tensors in device memory")
        # looked up where it is not the one before's: 16 states of one kind take 3 us less
        its = t.shape, t.stride(), t.dtype, t.device
        if its != kind:
            kind, ptrs = its, groups.setdefault(its, [])
        ptrs.append(t.data_ptr())
    for (shape, strides, dtype, device), ptrs in groups.items():
        if len(shape) < 2 or shape[0] != B or shape[1] != W:
            raise ValueError("a state must have shape [%d, %d, ...], got %s" % (B, W, tuple(shape)))
        if device != parent.device:
            raise ValueError("states must be on %s" % parent.device)
    layouts = [(_pieces(shape, strides, dtype.itemsize), ptrs) for (shape, strides, dtype, device), ptrs in groups.items() if 0 not in shape]
    torch.autograd.graph.increment_version(states)
    for layout, ptrs in layouts:
        _call("comet_beam_reorder", parent.device, stream, (ctypes.c_void_p * len(ptrs))(*ptrs), len(ptrs), B, W, *layout, parent.data_ptr())
