"""ctypes binding of libdolphin_hip.so: argument marshalling only.

Every function here has the name of the C entry point it calls (minus the
``dol_`` prefix where a class wraps a handle).  Device memory and the stream
come from PyTorch-ROCm; all arithmetic runs in the library's HIP kernels.
There is no fallback: if the shared library is missing, import fails.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdolphin_hip.so")

_NATIVE_PATH = os.path.join(_HERE, "_native.so")

if not (os.path.exists(LIB_PATH) and os.path.exists(_NATIVE_PATH)):
    raise ImportError(
        "libdolphin_hip.so or _native.so is not built (%s). Run `python -c 'import __graft_entry__ as g; g.build()'` "
        "or `python paper_2410_03348_amd/build.py`; there is no CPU fallback." % LIB_PATH)

_lib = C.CDLL(LIB_PATH)
from . import _native  # noqa: E402 (the calls issued once per operator; the others go through ctypes)

DAMP, DTKP = 0, 1
OP_APPLY2, OP_FILTER, OP_UNION, OP_FILTER_UNION = 0, 1, 2, 3
MAX_K, MAX_FACTS, MAX_SYMBOLS = 8, 63, 65535
ABSENT_PROOF = 0xFFFFFFFFFFFFFFFF
STATUS_NAMES = {0: "DOL_OK", 1: "DOL_EINVAL", 2: "DOL_ESHAPE", 3: "DOL_ENOMEM", 4: "DOL_EHIP", 5: "DOL_EUNSUPPORTED"}


class DolError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, str(status)), message))
        self.status = status


class _Prov(C.Structure):
    _fields_ = [("kind", C.c_int32), ("k", C.c_int32), ("n_facts", C.c_int32),
                ("fact_group", C.POINTER(C.c_int32)), ("fact_prob", C.c_void_p)]


class _Dist(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_sym", C.c_int32), ("ld", C.c_int64),
                ("sym_ids", C.POINTER(C.c_int32)), ("prob", C.c_void_p),
                ("proof_mask", C.c_void_p), ("proof_prob", C.c_void_p)]


class _OpRecord(C.Structure):
    _fields_ = [("op", C.c_int32), ("a", C.POINTER(_Dist)), ("b", C.POINTER(_Dist)), ("out", C.POINTER(_Dist)),
                ("f", C.c_void_p), ("pred_mask", C.POINTER(C.c_uint8)), ("prov", C.POINTER(_Prov)),
                ("accumulate", C.c_int32)]


_i32p = C.POINTER(C.c_int32)
_u8p = C.POINTER(C.c_uint8)
_lib.dol_fn_table_create_dense.argtypes = [C.c_int32, C.c_int32, _i32p, C.POINTER(C.c_void_p)]
_lib.dol_fn_table_create_sparse.argtypes = [C.c_int32, C.c_int32, C.c_int64, _i32p, _i32p, _i32p, C.POINTER(C.c_void_p)]
_lib.dol_fn_table_create_if.argtypes = [C.c_int32, C.c_int32, _i32p, _u8p, C.POINTER(C.c_void_p)]
_lib.dol_fnk_table_create.argtypes = [C.c_int32, _i32p, C.c_int64, _i32p, _i32p, C.POINTER(C.c_void_p)]
_lib.dol_fnk_table_n_out.argtypes = [C.c_void_p]
_lib.dol_fnk_table_n_out.restype = C.c_int32
_lib.dol_fnk_table_out_syms.argtypes = [C.c_void_p]
_lib.dol_fnk_table_out_syms.restype = _i32p
_lib.dol_fnk_table_kernel.argtypes = [C.c_void_p, C.c_int32]
_lib.dol_fnk_table_kernel.restype = C.c_char_p
_lib.dol_fnk_table_destroy.argtypes = [C.c_void_p]
_lib.dol_fnk_table_destroy.restype = None
_lib.dol_apply_k.argtypes = [C.c_int32, C.POINTER(C.POINTER(_Dist)), C.c_void_p, C.POINTER(_Prov), C.POINTER(_Dist), C.c_void_p]
_lib.dol_apply_k_backward.argtypes = [C.c_int32, C.POINTER(C.POINTER(_Dist)), C.c_void_p, C.POINTER(_Dist), C.c_void_p,
                                      C.c_int64, C.POINTER(C.c_void_p), C.c_void_p]
_lib.dol_fn_table_n_out.argtypes = [C.c_void_p]
_lib.dol_fn_table_n_out.restype = C.c_int32
_lib.dol_fn_table_out_syms.argtypes = [C.c_void_p]
_lib.dol_fn_table_out_syms.restype = _i32p
_lib.dol_fn_table_kernel.argtypes = [C.c_void_p, C.c_int32]
_lib.dol_fn_table_kernel.restype = C.c_char_p
_lib.dol_fn_table_kernel_at.argtypes = [C.c_void_p, C.c_int32, C.c_int64]
_lib.dol_fn_table_kernel_at.restype = C.c_char_p
_lib.dol_fn_table_destroy.argtypes = [C.c_void_p]
_lib.dol_fn_table_destroy.restype = None
_lib.dol_apply2.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.c_void_p, C.POINTER(_Prov), C.POINTER(_Dist), C.c_void_p]
_lib.dol_dtkp_apply2_input.argtypes = [C.POINTER(_Dist), _i32p, C.c_void_p, C.POINTER(_Prov), C.POINTER(_Dist), C.c_void_p]
_lib.dol_filter_plan.argtypes = [C.POINTER(_Dist), _u8p, _i32p, _i32p]
_lib.dol_filter.argtypes = [C.POINTER(_Dist), _u8p, C.POINTER(_Prov), C.POINTER(_Dist), C.c_void_p]
_lib.dol_union_plan.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), _i32p, _i32p]
_lib.dol_union.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.POINTER(_Prov), C.POINTER(_Dist), C.c_void_p]
_lib.dol_filter_union_plan.argtypes = [C.POINTER(_Dist), _u8p, C.POINTER(_Dist), _i32p, _i32p]
_lib.dol_filter_union.argtypes = [C.POINTER(_Dist), _u8p, C.POINTER(_Dist), C.POINTER(_Prov), C.POINTER(_Dist), C.c_void_p]
_lib.dol_dtkp_init.argtypes = [C.POINTER(_Dist), _i32p, C.POINTER(_Prov), C.c_void_p]
_lib.dol_backward.argtypes = [C.POINTER(_OpRecord), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dol_dtkp_backward.argtypes = [C.POINTER(_Dist), C.POINTER(_Prov), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
_lib.dol_nll_grad.argtypes = [C.POINTER(_Dist), C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dol_last_error.restype = C.c_char_p
_lib.dol_version.restype = C.c_char_p


def last_error() -> str:
    return _lib.dol_last_error().decode()


def version() -> str:
    return _lib.dol_version().decode()


def _check(status: int):
    if status != 0:
        raise DolError(status, last_error())


def _fail(status: int):
    raise DolError(status, last_error())


_native.setup(_fail, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, torch.float32, torch.bfloat16)


def _np_i32(x) -> np.ndarray:
    return np.ascontiguousarray(x, dtype=np.int32)


def _ptr(a: Optional[np.ndarray], ct):
    return None if a is None else a.ctypes.data_as(C.POINTER(ct))


def _handle(stream):
    """The same as the native calls take it: an integer, or None = torch's current stream."""
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else stream if stream is None else int(stream)


def _current() -> int:
    """The handle of torch's current stream alone: 0.2 us against 2.9 for a stream object, of 7 for a whole call."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream(stream) -> C.c_void_p:
    """A torch stream, a raw handle, or None = torch's current stream."""
    if stream is None:
        return C.c_void_p(_current())
    if isinstance(stream, torch.cuda.Stream):
        return C.c_void_p(stream.cuda_stream)
    return C.c_void_p(int(stream))


class Prov:
    """dol_prov.  fact_prob: float32 device tensor [batch, n_facts]; fact_group: host ints or None."""

    def __init__(self, kind: int = DAMP, k: int = 0, fact_prob: Optional[torch.Tensor] = None, fact_group=None):
        self.kind, self.k = kind, k
        self.fact_prob = fact_prob
        self._grp = None if fact_group is None else _np_i32(fact_group)
        n_facts = 0
        if fact_prob is not None:
            assert fact_prob.dtype == torch.float32 and fact_prob.is_contiguous() and fact_prob.dim() == 2
            n_facts = fact_prob.shape[1]
        if self._grp is not None:
            assert self._grp.size == n_facts
        self.c = _Prov(kind, k, n_facts, _ptr(self._grp, C.c_int32),
                       C.c_void_p(fact_prob.data_ptr()) if fact_prob is not None else None)
        self._p = C.addressof(self.c)

    def ref(self):
        return C.byref(self.c)


class Dist:
    """dol_dist over caller-owned torch tensors.  prob: float32 [batch, ld>=n_sym] (row stride = ld)."""

    def __init__(self, sym_ids, prob: Optional[torch.Tensor], proof_mask: Optional[torch.Tensor] = None,
                 proof_prob: Optional[torch.Tensor] = None, batch: Optional[int] = None):
        self.sym_ids = _np_i32(sym_ids)
        n = self.sym_ids.size
        self.prob, self.proof_mask, self.proof_prob = prob, proof_mask, proof_prob
        ld = n
        if prob is not None:
            assert prob.dtype == torch.float32 and prob.dim() == 2 and (prob.shape[1] == 0 or prob.stride(1) == 1)
            assert prob.shape[1] == n
            batch = prob.shape[0]
            ld = max(int(prob.stride(0)), n)
        for t, dt in ((proof_mask, (torch.int64, torch.uint64)), (proof_prob, (torch.float32,))):
            if t is not None:
                assert t.dtype in dt and t.is_contiguous() and t.dim() == 3 and t.shape[1] == n
                batch = t.shape[0] if batch is None else batch
        assert batch is not None
        self.batch, self.n_sym, self.ld = batch, n, ld
        self.c = _Dist(batch, n, ld, _ptr(self.sym_ids, C.c_int32),
                       C.c_void_p(prob.data_ptr()) if prob is not None else None,
                       C.c_void_p(proof_mask.data_ptr()) if proof_mask is not None else None,
                       C.c_void_p(proof_prob.data_ptr()) if proof_prob is not None else None)
        self._p = C.addressof(self.c)

    def ref(self):
        return C.byref(self.c)

    @staticmethod
    def empty(sym_ids, batch: int, device="cuda", k: int = 0, ld: Optional[int] = None) -> "Dist":
        """Allocate uninitialised tag tensors (torch is the allocator)."""
        n = len(sym_ids)
        ld = n if ld is None else ld
        prob = torch.empty((batch, ld), dtype=torch.float32, device=device)[:, :n] if ld != n else \
            torch.empty((batch, n), dtype=torch.float32, device=device)
        pm = pp = None
        if k > 0:
            pm = torch.empty((batch, n, k), dtype=torch.int64, device=device)
            pp = torch.empty((batch, n, k), dtype=torch.float32, device=device)
        return Dist(sym_ids, prob, pm, pp, batch=batch)


class FnTable:
    """dol_fn_table handle."""

    def __init__(self, handle: C.c_void_p, na: int, nb: int):
        self._h, self._p, self.na, self.nb = handle, handle.value, na, nb
        self.n_out = int(_lib.dol_fn_table_n_out(handle))
        p = _lib.dol_fn_table_out_syms(handle)
        self.out_syms = np.ctypeslib.as_array(p, shape=(self.n_out,)).copy() if self.n_out else np.empty(0, np.int32)
        self.kernel_fwd = _lib.dol_fn_table_kernel(handle, 0).decode()
        self.kernel_bwd = _lib.dol_fn_table_kernel(handle, 1).decode()

    def kernel_at(self, backward: bool, batch: int) -> str:
        """Name of the DAMP kernel launched for a batch of this size with contiguous, aligned tensors."""
        return _lib.dol_fn_table_kernel_at(self._h, 1 if backward else 0, batch).decode()

    @staticmethod
    def create_dense(out_id) -> "FnTable":
        t = _np_i32(out_id)
        assert t.ndim == 2
        h = C.c_void_p()
        _check(_lib.dol_fn_table_create_dense(t.shape[0], t.shape[1], _ptr(t, C.c_int32), C.byref(h)))
        return FnTable(h, t.shape[0], t.shape[1])

    @staticmethod
    def create_if(out_id, cond) -> "FnTable":
        """ApplyIf: the table of out_id restricted to the tuples where cond is non-zero."""
        t = _np_i32(out_id)
        c = np.ascontiguousarray(cond, dtype=np.uint8)
        assert t.ndim == 2 and c.shape == t.shape
        h = C.c_void_p()
        _check(_lib.dol_fn_table_create_if(t.shape[0], t.shape[1], _ptr(t, C.c_int32), _ptr(c, C.c_uint8), C.byref(h)))
        return FnTable(h, t.shape[0], t.shape[1])

    @staticmethod
    def create_sparse(na: int, nb: int, i, j, out_id) -> "FnTable":
        i, j, o = _np_i32(i), _np_i32(j), _np_i32(out_id)
        assert i.shape == j.shape == o.shape and i.ndim == 1
        h = C.c_void_p()
        _check(_lib.dol_fn_table_create_sparse(na, nb, i.size, _ptr(i, C.c_int32), _ptr(j, C.c_int32),
                                               _ptr(o, C.c_int32), C.byref(h)))
        return FnTable(h, na, nb)

    def destroy(self):
        if self._h is not None:
            _lib.dol_fn_table_destroy(self._h)
            self._h = self._p = None

    def __del__(self):
        # The collector may run this at any moment, also while a stream is being captured into a HIP graph, where
        # releasing device memory and code is not allowed: such handles wait for the next release outside a capture.
        try:
            if self._h is None:
                return
            if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
                _deferred_tables.append(self._h)
                self._h = self._p = None
                return
            self.destroy()
            while _deferred_tables:
                _lib.dol_fn_table_destroy(_deferred_tables.pop())
        except Exception:
            pass


_deferred_tables = []


def apply2(a: Dist, b: Dist, f: FnTable, prov: Optional[Prov], out: Dist, stream=None):
    _native.apply2(a._p, b._p, f._p, prov._p if prov else None, out._p, None if stream is None else _handle(stream))


class FnkTable:
    """dol_fnk_table handle: the admitted tuples of a function over K Distributions."""

    def __init__(self, n_sym, idx, out_id):
        n_sym, o = _np_i32(n_sym), _np_i32(out_id)
        self.K = int(n_sym.size)
        idx = _np_i32(idx).reshape(-1, self.K)
        assert idx.shape[0] == o.size
        h = C.c_void_p()
        _check(_lib.dol_fnk_table_create(self.K, _ptr(n_sym, C.c_int32), o.size, _ptr(idx, C.c_int32),
                                         _ptr(o, C.c_int32), C.byref(h)))
        self._h, self.n_sym = h, n_sym
        self.n_out = int(_lib.dol_fnk_table_n_out(h))
        self.kernel_fwd = _lib.dol_fnk_table_kernel(h, 0).decode()
        self.kernel_bwd = _lib.dol_fnk_table_kernel(h, 1).decode()
        p = _lib.dol_fnk_table_out_syms(h)
        self.out_syms = np.ctypeslib.as_array(p, shape=(self.n_out,)).copy() if self.n_out else np.empty(0, np.int32)

    @staticmethod
    def create_dense(out_id, cond=None) -> "FnkTable":
        """out_id: int array with one axis per operand; entries < 0, or where cond is zero, are rejected tuples."""
        t = _np_i32(out_id)
        if cond is not None:
            t = np.where(np.asarray(cond) != 0, t, -1).astype(np.int32)
        idx = np.argwhere(t >= 0).astype(np.int32).reshape(-1, t.ndim)
        return FnkTable(t.shape, idx, t[tuple(idx.T)])

    def destroy(self):
        if self._h is not None:
            _lib.dol_fnk_table_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _dist_array(dists):
    return (C.POINTER(_Dist) * len(dists))(*[C.pointer(d.c) for d in dists])


def apply_k(ins, f: FnkTable, prov: Optional[Prov], out: Dist, stream=None):
    _check(_lib.dol_apply_k(len(ins), _dist_array(ins), f._h, prov.ref() if prov else None, out.ref(), _stream(stream)))


def apply_k_backward(ins, f: FnkTable, out: Dist, grad_out: torch.Tensor, grad_in, stream=None):
    """grad_out [batch, >= n_out] (row stride = its stride(0)); grad_in: one tensor (rows of stride ins[l].ld) or None per operand."""
    assert grad_out.dtype == torch.float32 and grad_out.dim() == 2 and grad_out.stride(1) == 1
    ptrs = (C.c_void_p * len(ins))(*[None if g is None else g.data_ptr() for g in grad_in])
    _check(_lib.dol_apply_k_backward(len(ins), _dist_array(ins), f._h, out.ref(), _dptr(grad_out),
                                     max(int(grad_out.stride(0)), grad_out.shape[1]), ptrs, _stream(stream)))


def dtkp_apply2_input(a: Dist, fact_of_sym_b, f: FnTable, prov: Prov, out: Dist, stream=None):
    """dol_apply2 whose second operand is an input Distribution: symbol j of it is fact fact_of_sym_b[j]."""
    fb = _np_i32(fact_of_sym_b)
    assert fb.size == f.nb
    _native.dtkp_apply2_input(a._p, fb, f._p, prov._p, out._p, _handle(stream))


def filter_plan(d: Dist, pred_mask):
    pm = np.ascontiguousarray(pred_mask, dtype=np.uint8)
    n = C.c_int32()
    syms = np.empty(max(d.n_sym, 1), np.int32)
    _check(_lib.dol_filter_plan(d.ref(), _ptr(pm, C.c_uint8), C.byref(n), _ptr(syms, C.c_int32)))
    return syms[:n.value].copy()


def filter(d: Dist, pred_mask, prov: Optional[Prov], out: Dist, stream=None):  # noqa: A001 (the operator's name)
    pm = np.ascontiguousarray(pred_mask, dtype=np.uint8)
    _native.filter(d._p, pm, prov._p if prov else None, out._p, _handle(stream))


def union_plan(a: Dist, b: Dist):
    n = C.c_int32()
    syms = np.empty(max(a.n_sym + b.n_sym, 1), np.int32)
    _check(_lib.dol_union_plan(a.ref(), b.ref(), C.byref(n), _ptr(syms, C.c_int32)))
    return syms[:n.value].copy()


def union(a: Dist, b: Dist, prov: Optional[Prov], out: Dist, stream=None):
    _native.union(a._p, b._p, prov._p if prov else None, out._p, _handle(stream))


def filter_union_plan(d: Dist, pred_mask, c: Dist):
    pm = np.ascontiguousarray(pred_mask, dtype=np.uint8)
    n = C.c_int32()
    syms = np.empty(max(d.n_sym + c.n_sym, 1), np.int32)
    _check(_lib.dol_filter_union_plan(d.ref(), _ptr(pm, C.c_uint8), c.ref(), C.byref(n), _ptr(syms, C.c_int32)))
    return syms[:n.value].copy()


def filter_union(d: Dist, pred_mask, c: Dist, prov: Optional[Prov], out: Dist, stream=None):
    pm = np.ascontiguousarray(pred_mask, dtype=np.uint8)
    _check(_lib.dol_filter_union(d.ref(), _ptr(pm, C.c_uint8), c.ref(), prov.ref() if prov else None, out.ref(),
                                 _stream(stream)))


class _ApplyMerge(C.Structure):
    _fields_ = [("a", C.POINTER(_Dist)), ("b", C.POINTER(_Dist)), ("f", C.c_void_p), ("pred_mask", _u8p),
                ("c", C.POINTER(_Dist)), ("out", C.POINTER(_Dist)), ("saved", C.c_void_p)]


_lib.dol_apply2_filter_union.argtypes = [C.POINTER(_ApplyMerge), C.c_void_p]
_lib.dol_apply2_filter_union_backward.argtypes = [C.POINTER(_ApplyMerge), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                                  C.c_void_p, C.c_int32, C.c_void_p]
_lib.dol_apply2_filter_union_forward_backward.argtypes = _lib.dol_apply2_filter_union_backward.argtypes


class ApplyMerge:
    """dol_apply_merge: union(filter(apply2(a, b, f), pred_mask), c) described once, for the forward and reverse calls."""

    def __init__(self, a: Dist, b: Dist, f: FnTable, pred_mask, c: Dist, out: Dist, saved: Optional[torch.Tensor] = None):
        self._keep = (a, b, f, c, out, saved)
        self._pred = np.ascontiguousarray(pred_mask, dtype=np.uint8)
        assert self._pred.shape == (f.n_out,)
        assert saved is None or (saved.dtype == torch.int32 and saved.is_contiguous() and saved.shape == (a.batch,))
        self.c = _ApplyMerge(C.pointer(a.c), C.pointer(b.c), f._h, _ptr(self._pred, C.c_uint8), C.pointer(c.c), C.pointer(out.c),
                             C.c_void_p(saved.data_ptr()) if saved is not None else None)


def apply2_filter_union(m: ApplyMerge, stream=None):
    _check(_lib.dol_apply2_filter_union(C.byref(m.c), _stream(stream)))


def apply2_filter_union_backward(m: ApplyMerge, grad_out: torch.Tensor, grad_a: Optional[torch.Tensor],
                                 grad_b: Optional[torch.Tensor], grad_c: Optional[torch.Tensor], accumulate: int = 0,
                                 stream=None):
    assert grad_out.dtype == torch.float32 and grad_out.stride(1) == 1
    _check(_lib.dol_apply2_filter_union_backward(C.byref(m.c), _dptr(grad_out), int(grad_out.stride(0)), _dptr(grad_a),
                                                 _dptr(grad_b), _dptr(grad_c), accumulate, _stream(stream)))


def apply2_filter_union_forward_backward(m: ApplyMerge, grad_out: torch.Tensor, grad_a: Optional[torch.Tensor],
                                         grad_b: Optional[torch.Tensor], grad_c: Optional[torch.Tensor], accumulate: int = 0,
                                         stream=None):
    """Forward and backward of union(filter(apply2(a, b, f)), c) in one launch (grad_out is an input)."""
    assert grad_out.dtype == torch.float32 and grad_out.stride(1) == 1
    _check(_lib.dol_apply2_filter_union_forward_backward(C.byref(m.c), _dptr(grad_out), int(grad_out.stride(0)), _dptr(grad_a),
                                                         _dptr(grad_b), _dptr(grad_c), accumulate, _stream(stream)))


def dtkp_init(d: Dist, fact_of_sym, prov: Prov, stream=None):
    fos = _np_i32(fact_of_sym)
    _native.dtkp_init(d._p, fos, prov._p, _handle(stream))


class OpRecord:
    """dol_op_record; keeps its operands alive."""

    def __init__(self, op: int, a: Dist, b: Optional[Dist], out: Dist, f: Optional[FnTable] = None, pred_mask=None,
                 prov: Optional[Prov] = None, accumulate: int = 0):
        self.a, self.b, self.out, self.f, self.prov = a, b, out, f, prov
        self.pred = None if pred_mask is None else np.ascontiguousarray(pred_mask, dtype=np.uint8)
        self.c = _OpRecord(op, C.pointer(a.c), C.pointer(b.c) if b is not None else None, C.pointer(out.c),
                           f._h if f is not None else None, _ptr(self.pred, C.c_uint8),
                           C.pointer(prov.c) if prov is not None else None, accumulate)
        self._p = C.addressof(self.c)


def _dptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def backward(rec: OpRecord, grad_out: torch.Tensor, grad_a: Optional[torch.Tensor], grad_b: Optional[torch.Tensor],
             stream=None):
    """grad_out rows have stride rec.out.ld, grad_a rows rec.a.ld, grad_b rows rec.b.ld."""
    _native.backward(rec._p, None if grad_out is None else grad_out.data_ptr(), None if grad_a is None else grad_a.data_ptr(),
                     None if grad_b is None else grad_b.data_ptr(), None if stream is None else _handle(stream))


def dtkp_backward(d: Dist, prov: Prov, grad_prob: torch.Tensor, grad_fact_prob: torch.Tensor, stream=None):
    """grad_prob [batch, >= n_sym] (row stride = its stride(0)); grad_fact_prob [batch, n_facts] contiguous, overwritten."""
    assert grad_prob.dtype == torch.float32 and grad_prob.dim() == 2 and grad_prob.stride(1) == 1
    assert grad_fact_prob.dtype == torch.float32 and grad_fact_prob.is_contiguous()
    _native.dtkp_backward(d._p, prov._p, grad_prob.data_ptr(), max(int(grad_prob.stride(0)), grad_prob.shape[1]),
                          grad_fact_prob.data_ptr(), _handle(stream))


class _Fold(C.Structure):
    _fields_ = [("n_inputs", C.c_int32), ("inputs", C.POINTER(C.POINTER(_Dist))), ("tables", C.POINTER(C.c_void_p)),
                ("out", C.POINTER(_Dist)), ("target_col", C.c_void_p), ("grad_out", C.c_void_p),
                ("grad_out_ld", C.c_int64), ("grad_inputs", C.POINTER(C.c_void_p))]


_lib.dol_fold_apply2.argtypes = [C.POINTER(_Fold), C.c_void_p]
_lib.dol_fold_kernel.argtypes = [C.POINTER(_Fold)]
_lib.dol_fold_kernel.restype = C.c_char_p


class Fold:
    """dol_fold: a left fold of DAMP applies run forward (and backward) in one launch.  Keeps its operands alive."""

    def __init__(self, inputs, tables, out: Optional[Dist] = None, target_col: Optional[torch.Tensor] = None,
                 grad_out: Optional[torch.Tensor] = None, grad_inputs=None):
        n = len(inputs)
        assert len(tables) == n - 1
        self.keep = (inputs, tables, out, target_col, grad_out, grad_inputs)
        self._in = (C.POINTER(_Dist) * n)(*[C.pointer(d.c) for d in inputs])
        self._tb = (C.c_void_p * max(n - 1, 1))(*[t._h for t in tables])
        self._gi = None
        if grad_inputs is not None:
            assert len(grad_inputs) == n
            self._gi = (C.c_void_p * n)(*[None if g is None else g.data_ptr() for g in grad_inputs])
        if target_col is not None:
            assert target_col.dtype == torch.int32 and target_col.is_contiguous()
        ldg = 0
        if grad_out is not None:
            assert grad_out.dtype == torch.float32 and grad_out.dim() == 2 and grad_out.stride(1) == 1
            ldg = max(int(grad_out.stride(0)), grad_out.shape[1])
        self.c = _Fold(n, self._in, self._tb, C.pointer(out.c) if out is not None else None,
                       _dptr(target_col), _dptr(grad_out), ldg,
                       C.cast(self._gi, C.POINTER(C.c_void_p)) if self._gi is not None else None)
        self._p = C.addressof(self.c)


def fold_apply2(fold: Fold, stream=None):
    _native.fold_apply2(fold._p, None if stream is None else _handle(stream))


def fold_kernel(fold: Fold) -> str:
    return _lib.dol_fold_kernel(C.byref(fold.c)).decode()


class _DtkpFold(C.Structure):
    _fields_ = [("n_inputs", C.c_int32), ("inputs", C.POINTER(C.POINTER(_Dist))), ("fact_of_sym", C.POINTER(_i32p)),
                ("tables", C.POINTER(C.c_void_p)), ("out", C.POINTER(_Dist)), ("target_col", C.c_void_p),
                ("grad_out", C.c_void_p), ("grad_out_ld", C.c_int64), ("grad_fact_prob", C.c_void_p)]


_lib.dol_dtkp_fold_apply2.argtypes = [C.POINTER(_DtkpFold), C.POINTER(_Prov), C.c_void_p]
_lib.dol_dtkp_fold_kernel.argtypes = [C.POINTER(_DtkpFold), C.POINTER(_Prov)]
_lib.dol_dtkp_fold_kernel.restype = C.c_char_p


class DtkpFold:
    """dol_dtkp_fold: a left fold of DTKP applies over naturally initialised inputs, one launch.  Keeps its operands alive."""

    def __init__(self, inputs, facts, tables, out: Dist, target_col: Optional[torch.Tensor] = None,
                 grad_out: Optional[torch.Tensor] = None, grad_fact_prob: Optional[torch.Tensor] = None):
        n = len(inputs)
        assert len(tables) == n - 1 and len(facts) == n
        self._facts = [_np_i32(f) for f in facts]
        self.keep = (inputs, tables, out, target_col, grad_out, grad_fact_prob)
        self._in = (C.POINTER(_Dist) * n)(*[C.pointer(d.c) for d in inputs])
        self._fo = (_i32p * n)(*[_ptr(f, C.c_int32) for f in self._facts])
        self._tb = (C.c_void_p * max(n - 1, 1))(*[t._h for t in tables])
        if target_col is not None:
            assert target_col.dtype == torch.int32 and target_col.is_contiguous()
        ldg = 0
        if grad_out is not None:
            assert grad_out.dtype == torch.float32 and grad_out.dim() == 2 and grad_out.stride(1) == 1
            ldg = max(int(grad_out.stride(0)), grad_out.shape[1])
        if grad_fact_prob is not None:
            assert grad_fact_prob.dtype == torch.float32 and grad_fact_prob.is_contiguous()
        self.c = _DtkpFold(n, self._in, self._fo, self._tb, C.pointer(out.c), _dptr(target_col), _dptr(grad_out), ldg,
                           _dptr(grad_fact_prob))
        self._p = C.addressof(self.c)


def dtkp_fold_apply2(fold: DtkpFold, prov: Prov, stream=None):
    _native.dtkp_fold_apply2(fold._p, prov._p, None if stream is None else _handle(stream))


def dtkp_fold_kernel(fold: DtkpFold, prov: Prov) -> str:
    """Name of the kernel that dtkp_fold_apply2 launches for this fold."""
    return _lib.dol_dtkp_fold_kernel(C.byref(fold.c), C.byref(prov.c)).decode()


_lib.dol_iterate_apply2.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
_lib.dol_iterate_backward.argtypes = [C.POINTER(_Dist), C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64,
                                      C.c_void_p, C.c_void_p, C.c_void_p]


def iterate_apply2(r0: Dist, e: Dist, f: FnTable, rounds: int, hist: torch.Tensor, stream=None):
    """hist: float32 [rounds+1, batch, na] contiguous; receives r_0 .. r_rounds."""
    assert hist.dtype == torch.float32 and hist.is_contiguous() and hist.shape == (rounds + 1, r0.batch, f.na)
    _check(_lib.dol_iterate_apply2(r0.ref(), e.ref(), f._h, rounds, _dptr(hist), _stream(stream)))


def iterate_backward(e: Dist, f: FnTable, rounds: int, hist: torch.Tensor, grad_out: torch.Tensor,
                     grad_r0: Optional[torch.Tensor], grad_e: Optional[torch.Tensor], stream=None):
    """grad_out rows: stride grad_out.stride(0); grad_r0 [batch, na] contiguous; grad_e rows have stride e.ld."""
    assert hist.dtype == torch.float32 and hist.is_contiguous() and hist.shape == (rounds + 1, e.batch, f.na)
    assert grad_out.dtype == torch.float32 and grad_out.stride(1) == 1
    assert grad_r0 is None or grad_r0.is_contiguous()
    _check(_lib.dol_iterate_backward(e.ref(), f._h, rounds, _dptr(hist), _dptr(grad_out),
                                     max(int(grad_out.stride(0)), grad_out.shape[1]), _dptr(grad_r0), _dptr(grad_e),
                                     _stream(stream)))


_lib.dol_iterate_ckpt_count.argtypes = [C.c_int32, C.c_int32]
_lib.dol_iterate_ckpt_count.restype = C.c_int32
_lib.dol_iterate_ckpt_every.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
_lib.dol_iterate_ckpt_every.restype = C.c_int32
_lib.dol_iterate_kernel.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
_lib.dol_iterate_kernel.restype = C.c_char_p
_lib.dol_iterate_apply2_ckpt.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.c_void_p, C.c_int32, C.c_int32,
                                         C.POINTER(_Dist), C.c_void_p, C.c_void_p]
_lib.dol_iterate_backward_ckpt.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.c_void_p, C.c_int32, C.c_int32,
                                           C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]


def iterate_ckpt_count(rounds: int, ckpt_every: int) -> int:
    return int(_lib.dol_iterate_ckpt_count(rounds, ckpt_every))


def iterate_ckpt_every(f: FnTable, batch: int, rounds: int) -> int:
    """The checkpoint interval the library favours for this table, batch and round count."""
    return int(_lib.dol_iterate_ckpt_every(f._h, batch, rounds))


def iterate_kernel(f: FnTable, batch: int, rounds: int, ckpt_every: int) -> str:
    """The kernel that iterate_apply2_backward launches; "" where its sweeps are two launches."""
    return _lib.dol_iterate_kernel(f._h, batch, rounds, ckpt_every).decode()


def iterate_apply2_ckpt(r0: Dist, e: Dist, f: FnTable, rounds: int, ckpt_every: int, out: Dist,
                        ckpt: Optional[torch.Tensor], stream=None):
    """ckpt: float32 [iterate_ckpt_count(rounds, ckpt_every), batch, na] contiguous (None when that count is 0)."""
    n = iterate_ckpt_count(rounds, ckpt_every)
    assert n == 0 or (ckpt.dtype == torch.float32 and ckpt.is_contiguous() and ckpt.shape == (n, r0.batch, f.na))
    _check(_lib.dol_iterate_apply2_ckpt(r0.ref(), e.ref(), f._h, rounds, ckpt_every, out.ref(), _dptr(ckpt),
                                        _stream(stream)))


def iterate_backward_ckpt(r0: Dist, e: Dist, f: FnTable, rounds: int, ckpt_every: int, ckpt: Optional[torch.Tensor],
                          grad_out: torch.Tensor, grad_r0: Optional[torch.Tensor], grad_e: Optional[torch.Tensor],
                          stream=None):
    assert grad_out.dtype == torch.float32 and grad_out.stride(1) == 1
    assert grad_r0 is None or grad_r0.is_contiguous()
    _check(_lib.dol_iterate_backward_ckpt(r0.ref(), e.ref(), f._h, rounds, ckpt_every, _dptr(ckpt), _dptr(grad_out),
                                          max(int(grad_out.stride(0)), grad_out.shape[1]), _dptr(grad_r0), _dptr(grad_e),
                                          _stream(stream)))


_lib.dol_iterate_apply2_backward.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.c_void_p, C.c_int32, C.c_int32,
                                             C.POINTER(_Dist), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                             C.c_void_p, C.c_void_p]


def iterate_apply2_backward(r0: Dist, e: Dist, f: FnTable, rounds: int, ckpt_every: int, out: Dist,
                            ckpt: Optional[torch.Tensor], target_col: Optional[torch.Tensor], grad_out: Optional[torch.Tensor],
                            grad_r0: Optional[torch.Tensor], grad_e: Optional[torch.Tensor], stream=None):
    """Forward rounds and reverse sweep in one call (one launch up to 512 samples); exactly one of target_col (int32 [batch])
    and grad_out."""
    ldg = 0
    if grad_out is not None:
        assert grad_out.dtype == torch.float32 and grad_out.stride(1) == 1
        ldg = max(int(grad_out.stride(0)), grad_out.shape[1])
    if target_col is not None:
        assert target_col.dtype == torch.int32 and target_col.is_contiguous()
    assert grad_r0 is None or grad_r0.is_contiguous()
    _check(_lib.dol_iterate_apply2_backward(r0.ref(), e.ref(), f._h, rounds, ckpt_every, out.ref(), _dptr(ckpt), _dptr(target_col),
                                            _dptr(grad_out), ldg, _dptr(grad_r0), _dptr(grad_e), _stream(stream)))


_lib.dol_iterate_backward_noalloc.argtypes = [C.POINTER(_Dist), C.POINTER(_Dist), C.c_void_p, C.c_int32, C.c_void_p,
                                              C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]


def iterate_backward_noalloc(r0: Dist, e: Dist, f: FnTable, rounds: int, grad_out: torch.Tensor,
                             grad_r0: Optional[torch.Tensor], grad_e: Optional[torch.Tensor], stream=None):
    """The reverse sweep with the library's built-in workspace: no allocation, forward sweep replayed inside."""
    assert grad_out.dtype == torch.float32 and grad_out.stride(1) == 1
    assert grad_r0 is None or grad_r0.is_contiguous()
    _check(_lib.dol_iterate_backward_noalloc(r0.ref(), e.ref(), f._h, rounds, _dptr(grad_out),
                                             max(int(grad_out.stride(0)), grad_out.shape[1]), _dptr(grad_r0),
                                             _dptr(grad_e), _stream(stream)))


def nll_grad(d: Dist, target_col: torch.Tensor, grad: torch.Tensor, stream=None):
    """target_col: int32 device tensor [batch]; grad rows have stride d.ld."""
    assert target_col.dtype == torch.int32 and target_col.is_contiguous()
    _native.nll_grad(d._p, target_col.data_ptr(), grad.data_ptr(), None if stream is None else _handle(stream))


# ---- training the network whose outputs become Distributions

F32, BF16 = 0, 1
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


# The calls below check tensors and take them apart in _native: matrix(t) and activations(t) give the fields of the structures,
# values(t, dtype, sizes..) the address of a contiguous tensor, all of them None for None; AssertionError where a tensor does not fit.
_matrix, _activations, _values = _native.matrix, _native.activations, _native.values
_F, _I = torch.float32, torch.int32


def _workspace(given: Optional[torch.Tensor], n: int, device, stream):
    """(address, bytes, what keeps it): the caller's workspace, or n bytes of torch's allocator.  Those are taken on the stream that the call
    is on: whoever had them before and has them after is on it too, while work of the current stream may still use what that one freed."""
    if given is not None:
        assert given.is_cuda and given.is_contiguous()
        return given.data_ptr(), given.numel() * given.element_size(), given
    if n == 0:
        return None, 0, None
    if stream is None or _handle(stream) == _current():
        t = torch.empty(n, dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=device)):
            t = torch.empty(n, dtype=torch.uint8, device=device)
    return t.data_ptr(), n, t


def cross_entropy_workspace(x: torch.Tensor, weight: torch.Tensor, backward: bool = False) -> int:
    """Bytes that cross_entropy (or cross_entropy_backward) needs for these operands."""
    return _native.cross_entropy_workspace(_matrix(x), _matrix(weight), int(backward))


def cross_entropy_kernel(x: torch.Tensor, weight: torch.Tensor, backward: bool = False) -> str:
    """The kernels that multiply for these operands, and their tiles."""
    return _native.cross_entropy_kernel(_matrix(x), _matrix(weight), int(backward))


def cross_entropy(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, loss: torch.Tensor, lse: torch.Tensor,
                  bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """loss[i] = lse[i] - (x[i] . weight[target[i]] + bias[target[i]]), lse the log of the sum of the exponentials over all classes.

    x [rows, width], weight [classes, width] (float32 or bfloat16); target int32 [rows], rows outside 0..classes-1 are left out;
    loss, lse float32 [rows]; bias float32 [classes]; workspace: any tensor of cross_entropy_workspace bytes, or None."""
    mx, mw = _matrix(x), _matrix(weight)
    rows, classes = mx[1], mw[1]
    ws, n, _keep = _workspace(workspace, _native.cross_entropy_workspace(mx, mw, 0) if workspace is None else 0, x.device, stream)
    _native.cross_entropy(mx, mw, _values(bias, _F, classes), _values(target, _I, rows), _values(loss, _F, rows), _values(lse, _F, rows),
                          ws, n, _handle(stream))


def cross_entropy_backward(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, lse: torch.Tensor, grad_loss: torch.Tensor,
                           grad_x: Optional[torch.Tensor], grad_weight: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                           grad_bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of sum_i grad_loss[i] loss[i]; lse as cross_entropy left it.  Gradients that are None are not computed."""
    mx, mw = _matrix(x), _matrix(weight)
    rows, classes = mx[1], mw[1]
    ws, n, _keep = _workspace(workspace, _native.cross_entropy_workspace(mx, mw, 1) if workspace is None else 0, x.device, stream)
    _native.cross_entropy_backward(mx, mw, _values(bias, _F, classes), _values(target, _I, rows), _values(lse, _F, rows),
                                   _values(grad_loss, _F, rows), _matrix(grad_x), _matrix(grad_weight), _values(grad_bias, _F, classes),
                                   ws, n, _handle(stream))


def _matrices(t: torch.Tensor):
    """(the first matrix, elements from one to the next, how many) of a tensor [rows, cols] or [batch, rows, cols]."""
    if t.dim() == 2:
        return _matrix(t), 0, 1
    assert t.dim() == 3
    b, rows, cols = t.shape
    assert t.is_cuda and t.dtype in _DTYPES and (cols <= 1 or t.stride(2) == 1) and (rows <= 1 or t.stride(1) >= cols)
    return (_DTYPES[t.dtype], rows, cols, t.stride(1) if rows > 1 else max(cols, 1), t.data_ptr()), t.stride(0), b


def newton_schulz_workspace(g: torch.Tensor) -> int:
    m, _, batch = _matrices(g)
    return _native.newton_schulz_workspace(m, batch)


def newton_schulz_kernel(g: torch.Tensor) -> str:
    """The kernels that multiply for these matrices, and their tiles."""
    m, _, batch = _matrices(g)
    return _native.newton_schulz_kernel(m, batch)


def newton_schulz(g: torch.Tensor, out: torch.Tensor, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  workspace: Optional[torch.Tensor] = None, stream=None):
    """out = X after `steps` times X <- a X + (b A + c A A) X, A = X X^T, from X = g / (|g| + eps): g's singular vectors with singular
    values near 1.  g, out: [rows, cols] or [batch, rows, cols], float32 or bfloat16; out may be g."""
    mg, g_stride, batch = _matrices(g)
    mo, out_stride, n_out = _matrices(out)
    assert batch == n_out
    ws, n, _keep = _workspace(workspace, _native.newton_schulz_workspace(mg, batch) if workspace is None else 0, g.device, stream)
    _native.newton_schulz(mg, g_stride, mo, out_stride, batch, steps, *coefficients, eps, ws, n, _handle(stream))


_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def group_norm_workspace(x: torch.Tensor, groups: int, backward: bool = False) -> int:
    return _native.group_norm_workspace(_activations(x), groups, int(backward))


def group_norm(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], groups: int, y: torch.Tensor,
               mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor], eps: float = 1e-5, act: str = "none",
               workspace: Optional[torch.Tensor] = None, stream=None):
    """y = act(gamma * (x - mean) * rstd + beta), mean and variance over the points of a sample and the channels of a group.

    x, y: [batch, points.., channels] (float32 or bfloat16; y may be x); gamma, beta: float32 [channels]; mean, rstd: float32
    [batch, groups], written; act: "none", "relu", "silu" or "gelu"."""
    mx = _activations(x)
    batch, channels = mx[1], mx[3]
    ws, n, _keep = _workspace(workspace, _native.group_norm_workspace(mx, groups, 0) if workspace is None else 0, x.device, stream)
    _native.group_norm(mx, groups, _values(gamma, _F, channels), _values(beta, _F, channels), eps, _ACTS[act], _activations(y),
                       _values(mean, _F, batch, groups), _values(rstd, _F, batch, groups), ws, n, _handle(stream))


def group_norm_backward(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], groups: int, mean: torch.Tensor,
                        rstd: torch.Tensor, grad_y: torch.Tensor, grad_x: Optional[torch.Tensor], grad_gamma: Optional[torch.Tensor],
                        grad_beta: Optional[torch.Tensor], act: str = "none", workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of sum(grad_y * y); mean and rstd as group_norm left them.  Gradients that are None are not computed; grad_x may be
    grad_y or x."""
    mx = _activations(x)
    batch, channels = mx[1], mx[3]
    ws, n, _keep = _workspace(workspace, _native.group_norm_workspace(mx, groups, 1) if workspace is None else 0, x.device, stream)
    _native.group_norm_backward(mx, groups, _values(gamma, _F, channels), _values(beta, _F, channels), _ACTS[act],
                                _values(mean, _F, batch, groups), _values(rstd, _F, batch, groups), _activations(grad_y),
                                _activations(grad_x), _values(grad_gamma, _F, channels), _values(grad_beta, _F, channels), ws, n,
                                _handle(stream))


def linear_workspace(x: torch.Tensor, weight: torch.Tensor, backward: bool = False) -> int:
    """Bytes that linear (or linear_backward) needs for these operands."""
    return _native.linear_workspace(_matrix(x), _matrix(weight), int(backward))


def linear_kernel(x: torch.Tensor, weight: torch.Tensor, backward: bool = False) -> str:
    """The kernel that multiplies for these operands, and its tiles."""
    return _native.linear_kernel(_matrix(x), _matrix(weight), int(backward))


def linear(x: torch.Tensor, weight: torch.Tensor, y: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
           residual: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None, z_rest: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, stream=None):
    """y = act(z) + residual, z = x weight^T + bias.

    x [rows, width], weight [out, width] (float32 or bfloat16); y, residual, z [rows, out] of that type, y may be the residual; bias float32
    [out]; act: "none", "relu", "silu" or "gelu".  The gradients need z where act is not "none"; z_rest int16 [rows, out], beside a z in bfloat16,
    keeps grad_bias as exact as sums in 32 bits, at no cost in time: training in bfloat16 wants it.  Without it grad_bias is off by 6e-4 or so."""
    mx, mw = _matrix(x), _matrix(weight)
    rows, out = mx[1], mw[1]
    ws, n, _keep = _workspace(workspace, _native.linear_workspace(mx, mw, 0) if workspace is None else 0, x.device, stream)
    _native.linear(mx, mw, _values(bias, _F, out), _ACTS[act], _matrix(residual), _matrix(y), _matrix(z), _values(z_rest, torch.int16, rows, out), ws, n,
                   _handle(stream))


def linear_backward(x: torch.Tensor, weight: torch.Tensor, grad_y: torch.Tensor, grad_x: Optional[torch.Tensor],
                    grad_weight: Optional[torch.Tensor], grad_bias: Optional[torch.Tensor] = None, act: str = "none",
                    z: Optional[torch.Tensor] = None, z_rest: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None):
    """Gradients of sum(grad_y * y); z and z_rest as linear left them.  Gradients that are None are not computed; the residual's is grad_y."""
    mx, mw = _matrix(x), _matrix(weight)
    rows, out = mx[1], mw[1]
    ws, n, _keep = _workspace(workspace, _native.linear_workspace(mx, mw, 1) if workspace is None else 0, x.device, stream)
    _native.linear_backward(mx, mw, _ACTS[act], _matrix(z), _values(z_rest, torch.int16, rows, out), _matrix(grad_y), _matrix(grad_x),
                            _matrix(grad_weight), _values(grad_bias, _F, out), ws, n, _handle(stream))


def residual_norm(x: Optional[torch.Tensor], u: torch.Tensor, gamma_u: Optional[torch.Tensor], gate: Optional[torch.Tensor],
                  gamma_y: Optional[torch.Tensor], h: Optional[torch.Tensor], y: Optional[torch.Tensor], rstd_u: Optional[torch.Tensor] = None,
                  rstd_h: Optional[torch.Tensor] = None, norm_u: bool = True, scale: float = 1.0, eps: float = 1e-6, stream=None):
    """h = x + scale * gate * v, v = gamma_u * u * rstd_u (u itself without norm_u); y = gamma_y * h * rstd_h; rstd of a row = 1 / sqrt(mean of
    its squares + eps).

    x (None = 0), u, h, y: [rows, cols] (float32 or bfloat16; h and y may be x or u, either may be None); gate: [gates, cols] of that type, where
    gates divides rows and each gate serves rows / gates neighbours; gamma_u, gamma_y: float32 [cols]; rstd_u, rstd_h: float32 [rows], written."""
    mu = _matrix(u)
    rows, cols = mu[1], mu[2]
    _native.residual_norm(_matrix(x), mu, int(norm_u), _values(gamma_u, _F, cols), _matrix(gate), scale, _values(gamma_y, _F, cols), eps, _matrix(h),
                          _matrix(y), _values(rstd_u, _F, rows), _values(rstd_h, _F, rows), _handle(stream))


def residual_norm_workspace(u: torch.Tensor, gate: Optional[torch.Tensor] = None) -> int:
    """Bytes that residual_norm_backward needs for these operands; residual_norm needs none."""
    return _native.residual_norm_workspace(_matrix(u), _matrix(gate))


def residual_norm_backward(x: Optional[torch.Tensor], u: torch.Tensor, gamma_u: Optional[torch.Tensor], gate: Optional[torch.Tensor],
                           gamma_y: Optional[torch.Tensor], rstd_u: Optional[torch.Tensor], rstd_h: Optional[torch.Tensor],
                           grad_h: Optional[torch.Tensor], grad_y: Optional[torch.Tensor], grad_x: Optional[torch.Tensor],
                           grad_u: Optional[torch.Tensor], grad_gamma_u: Optional[torch.Tensor], grad_gate: Optional[torch.Tensor],
                           grad_gamma_y: Optional[torch.Tensor], norm_u: bool = True, scale: float = 1.0,
                           workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of sum(grad_h * h) + sum(grad_y * y); rstd_u and rstd_h as residual_norm left them.  Gradients that are None are not
    computed; grad_x and grad_u may be grad_h, grad_y, x or u, but not one tensor.

    A program that keeps h and not x calls residual_norm_backward(u, gamma_u, gate, gamma_y, h, rstd_u, ...), the same from there on: with h behind
    gamma_y in place of x before u, which the vector gamma_u (or None) in the place of the matrix u tells apart.  In bfloat16 grad_gamma_y is then
    off by what rounding h has left, some 2^-9 a term."""
    call = _native.residual_norm_backward
    if u is None or u.dim() == 1:
        x, u, gamma_u, gate, gamma_y = gamma_y, x, u, gamma_u, gate
        call = _native.residual_norm_backward_from_h
    mu, mg = _matrix(u), _matrix(gate)
    rows, cols = mu[1], mu[2]
    ws, n, _keep = _workspace(workspace, _native.residual_norm_workspace(mu, mg) if workspace is None else 0, u.device, stream)
    call(_matrix(x), mu, int(norm_u), _values(gamma_u, _F, cols), mg, scale, _values(gamma_y, _F, cols), _values(rstd_u, _F, rows),
         _values(rstd_h, _F, rows), _matrix(grad_h), _matrix(grad_y), _matrix(grad_x), _matrix(grad_u), _values(grad_gamma_u, _F, cols),
         _matrix(grad_gate), _values(grad_gamma_y, _F, cols), ws, n, _handle(stream))


_lib.dol_tensor_list_create.argtypes = [C.c_int32, _i32p, C.POINTER(C.c_int64), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p)]
_lib.dol_tensor_list_destroy.argtypes = [C.c_void_p]
_lib.dol_tensor_list_destroy.restype = None


def _dense(t: torch.Tensor) -> bool:
    """Whether the tensor's elements fill one stretch of memory, in whatever order its dimensions lie."""
    want = 1
    for stride, size in sorted((st, n) for n, st in zip(t.shape, t.stride()) if n != 1):
        if stride != want:
            return t.numel() == 0
        want *= size
    return True


class TensorList:
    """The buffers of a network's gradients, in the order given: float32 or bfloat16 tensors of one device, each without gaps in memory.
    Keeps the tensors, whose memory the calls use; made once for buffers that a program keeps."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        n = len(self.tensors)
        dtype, size, data = (C.c_int32 * max(n, 1))(), (C.c_int64 * max(n, 1))(), (C.c_void_p * max(n, 1))()
        for k, t in enumerate(self.tensors):
            assert t.is_cuda and t.device == self.tensors[0].device and t.dtype in _DTYPES and _dense(t)
            dtype[k], size[k], data[k] = _DTYPES[t.dtype], t.numel(), t.data_ptr()
        self.device = self.tensors[0].device if n else None
        # two lists whose tensors lie in memory in another order are not each other's results; None = the order of the dimensions
        self._orders = None if all(t.is_contiguous() for t in self.tensors) else [(tuple(t.shape), t.stride()) for t in self.tensors]
        self._h = None
        h = C.c_void_p()
        with torch.cuda.device(self.device) if n else contextlib.nullcontext():
            _check(_lib.dol_tensor_list_create(n, dtype, size, data, C.byref(h)))
        self._h = h.value

    def destroy(self):
        if self._h:
            _lib.dol_tensor_list_destroy(self._h)
            self._h = None

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            self.destroy()


def grad_norm_workspace(grads: TensorList) -> int:
    """Bytes that grad_norm and clip_grads need for this list."""
    return _native.grad_norm_workspace(grads._h)


def grad_norm(grads: TensorList, norm: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None):
    """norm float32 [1]: the root of the sum of the squares of all elements of all tensors."""
    ws, n, _keep = _workspace(workspace, _native.grad_norm_workspace(grads._h) if workspace is None else 0, norm.device, stream)
    _native.grad_norm(grads._h, _values(norm, _F, 1), ws, n, _handle(stream))


def clip_grads(grads: TensorList, max_norm: float, norm: torch.Tensor, coef: torch.Tensor, out: Optional[TensorList] = None, eps: float = 1e-6,
               workspace: Optional[torch.Tensor] = None, stream=None):
    """out = coef * grads (None: in place), coef = min(1, max_norm / (norm + eps)), norm as grad_norm gives it; norm, coef: float32 [1]."""
    out = grads if out is None else out
    assert out is grads or out._orders == grads._orders
    ws, n, _keep = _workspace(workspace, _native.grad_norm_workspace(grads._h) if workspace is None else 0, norm.device, stream)
    _native.clip_grads(grads._h, out._h, max_norm, eps, _values(norm, _F, 1), _values(coef, _F, 1), ws, n, _handle(stream))
