"""Binding of the attention calls (dsv_attn_* of include/dsv.h): argument marshalling only.

One plan holds a mixed batch's sequences -- whole prompts, chunks behind a cached prefix, single decode tokens and
fine-tuning samples -- and serves every layer:

    plan = attn.Plan([(q_start, q_len, k_start, k_len, is_train), ...], n_q, n_kv, heads_q, heads_kv, head_dim,
                     device="cuda")
    O, lse = attn.fwd(plan, Q, K, V)                      # Q [n_q][heads_q][d]; K, V [n_kv][heads_kv][d]
    dQ, dK, dV = attn.bwd(plan, Q, K, V, O, lse, dO)      # rows of the fine-tuning samples alone ("compact order")

Query i of a sequence sees its keys j <= i + k_len - q_len.  Tensors may be any views whose head vectors are
contiguous, but not broadcast ones: columns of a q/k/v product, a cache laid out [row][head][d] or [head][row][d].
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import struct

import numpy as np

from . import dsv
from .dsv import DsvError, _check, _ptr, _stream_handle, torch  # noqa: F401

_lib = dsv.lib_handle()
_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t


class View(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("row", _i64), ("head", _i64)]


_viewp = ctypes.POINTER(View)
_lib.dsv_attn_build.argtypes = [_vp, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(_sz), ctypes.POINTER(_vp)]
_lib.dsv_attn_build.restype = ctypes.c_int
_lib.dsv_attn_upload.argtypes = [_vp, _vp, _sz, _vp]
_lib.dsv_attn_upload.restype = ctypes.c_int
_lib.dsv_attn_train_rows.argtypes = [_vp, ctypes.POINTER(_i64)]
_lib.dsv_attn_train_rows.restype = ctypes.c_int
_lib.dsv_attn_free.argtypes = [_vp]
_lib.dsv_attn_free.restype = None
_lib.dsv_attn_workspace.argtypes = [_vp, ctypes.c_int, ctypes.POINTER(_sz)]
_lib.dsv_attn_workspace.restype = ctypes.c_int
_lib.dsv_attn_fwd.argtypes = [_vp, ctypes.c_int, ctypes.c_double] + [_viewp] * 4 + [_vp, _vp, _sz, _vp]
_lib.dsv_attn_fwd.restype = ctypes.c_int
_lib.dsv_attn_bwd.argtypes = [_vp, ctypes.c_int, ctypes.c_double] + [_viewp] * 4 + [_vp] + [_viewp] * 4 + [_vp, _sz, _vp]
_lib.dsv_attn_bwd.restype = ctypes.c_int

# The calls below pass their views as packed bytes, read during the call only: a decode step's attention takes the GPU
# 10 us, and marshalling structures takes the host as long.
_VIEW_PACK = struct.Struct("@Pqq").pack
assert len(_VIEW_PACK(0, 0, 0)) == ctypes.sizeof(View)
_head = (ctypes.c_int, _vp, ctypes.c_int, ctypes.c_double)
_fwd = ctypes.CFUNCTYPE(*_head, *[_vp] * 6, _sz, _vp)(("dsv_attn_fwd", _lib))
_bwd = ctypes.CFUNCTYPE(*_head, *[_vp] * 10, _sz, _vp)(("dsv_attn_bwd", _lib))


def on(stream):
    """Where a call allocates what it was not given: on the call's stream, so that neither the memory's earlier use nor
    its filling runs beside the call."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def int32(**named):
    """The numbers, in order; ValueError for one that the library, which takes 32 bits of it, would see cut off."""
    for name, x in named.items():
        if not -(1 << 31) <= int(x) < 1 << 31:
            raise ValueError("%s = %d does not fit 32 bits" % (name, x))
    return [int(x) for x in named.values()]


class Plan:
    """The packed sequences of a batch.  device=None builds a host-only plan (inspection only)."""

    def __init__(self, seqs, n_q: int, n_kv: int, heads_q: int, heads_kv: int, head_dim: int, device=None, stream=None):
        table = np.asarray(seqs).reshape(-1, 5)
        if not np.all((table >= -(1 << 31)) & (table < 1 << 31)):
            raise ValueError("seqs holds numbers that do not fit 32 bits")
        self.seqs = np.ascontiguousarray(table, np.int32)
        self.n_q, self.n_kv, self.heads_q, self.heads_kv, self.head_dim = int32(
            n_q=n_q, n_kv=n_kv, heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim)
        self._h = _vp()
        self.meta = None
        n = _sz(0)
        _check(_lib.dsv_attn_build(self.seqs.ctypes.data, self.seqs.shape[0], self.n_q, self.n_kv, self.heads_q,
                                   self.heads_kv, self.head_dim, ctypes.byref(n), ctypes.byref(self._h)),
               "dsv_attn_build")
        self.meta_bytes = int(n.value)
        rows = (_i64 * 2)()
        _check(_lib.dsv_attn_train_rows(self._h, rows), "dsv_attn_train_rows")
        self.train_q, self.train_k = int(rows[0]), int(rows[1])
        if device is not None:
            with on(stream):
                self.meta = torch.empty(self.meta_bytes, dtype=torch.uint8, device=device)
            _check(_lib.dsv_attn_upload(self._h, _ptr(self.meta), n, _stream_handle(stream)), "dsv_attn_upload")

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:  # _lib is None at interpreter exit
            _lib.dsv_attn_free(h)
            self._h = _vp()

    @property
    def handle(self):
        return self._h


def _code(dtype) -> int:
    if dtype == torch.bfloat16:
        return dsv.BF16
    if dtype == torch.float32:
        return dsv.F32
    raise TypeError("dsv supports bfloat16 and float32 tensors, got %s" % dtype)


def workspace_bytes(plan: Plan, dtype) -> int:
    """Bytes of device workspace for fwd and bwd of this plan (one buffer serves both)."""
    n = _sz(0)
    _check(_lib.dsv_attn_workspace(plan.handle, _code(dtype), ctypes.byref(n)), "dsv_attn_workspace")
    return int(n.value)


def _view(t, rows: int, heads: int, d: int, dtype, name: str) -> bytes:
    if t.dtype is not dtype:
        raise TypeError("%s is %s, the call's tensors are %s" % (name, t.dtype, dtype))
    if t.shape != (rows, heads, d):
        if t.shape != (rows, heads * d):
            raise ValueError("%s must be [%d][%d][%d], got %s" % (name, rows, heads, d, tuple(t.shape)))
        t = t.unflatten(1, (heads, d))
    row, head, one = t.stride()
    if one != 1 and rows:
        raise ValueError("%s: the elements of a head must be contiguous" % name)
    # the library takes a stride of 0 for the dense one
    if (row == 0 and rows > 1) or (head == 0 and heads > 1 and rows > 0):
        raise ValueError("%s is broadcast (a stride of 0): make it contiguous" % name)
    # a stride of a dimension of one is arbitrary: the dense one then
    return _VIEW_PACK(t.data_ptr(), row if rows > 1 else 0, head if heads > 1 and rows > 0 else 0)


def _dense(t, shape, name: str):
    if t.dtype is not torch.float32 or not t.is_contiguous() or t.shape != shape:
        raise ValueError("%s must be a contiguous fp32 tensor of shape %s" % (name, shape))
    return t.data_ptr()


def _ws(given, plan, like, stream):
    if given is not None:
        return given
    with on(stream):
        return torch.empty(workspace_bytes(plan, like.dtype), dtype=torch.uint8, device=like.device)


def fwd(plan: Plan, Q, K, V, scale=None, O=None, lse=None, want_lse=None, workspace=None, stream=None):
    """dsv_attn_fwd; returns (O, lse).  scale: 1 / sqrt(head_dim) if None.  lse is [heads_q][n_q] fp32, which a backward
    needs; without one it is made if want_lse, which stands for "where O is made" if None, else it is not written and
    None is returned for it (inference)."""
    hq, hkv, d = plan.heads_q, plan.heads_kv, plan.head_dim
    make_lse = lse is None and (O is None if want_lse is None else want_lse)
    if O is None or make_lse:
        with on(stream):
            # rows that no sequence holds are not written
            if O is None:
                O = torch.zeros((plan.n_q, hq, d), dtype=Q.dtype, device=Q.device)
            if make_lse:
                lse = torch.full((hq, plan.n_q), -math.inf, dtype=torch.float32, device=Q.device)
    ws, dt = _ws(workspace, plan, Q, stream), Q.dtype
    _check(_fwd(plan.handle, _code(dt), 1 / math.sqrt(d) if scale is None else scale,
                _view(Q, plan.n_q, hq, d, dt, "Q"), _view(K, plan.n_kv, hkv, d, dt, "K"),
                _view(V, plan.n_kv, hkv, d, dt, "V"), _view(O, plan.n_q, hq, d, dt, "O"),
                None if lse is None else _dense(lse, (hq, plan.n_q), "lse"), ws.data_ptr(), ws.nbytes,
                _stream_handle(stream)), "dsv_attn_fwd")
    return O, lse


def bwd(plan: Plan, Q, K, V, O, lse, dO, scale=None, dQ=None, dK=None, dV=None, workspace=None, stream=None):
    """dsv_attn_bwd; returns (dQ, dK, dV): [train_q][heads_q][d] and twice [train_k][heads_kv][d].  lse: the forward's
    (None only where the plan has no fine-tuning rows)."""
    hq, hkv, d, nq, nk = plan.heads_q, plan.heads_kv, plan.head_dim, plan.train_q, plan.train_k
    if lse is None and nq > 0:
        raise ValueError("lse is None: the forward returns it with lse=... or want_lse=True")
    if dQ is None or dK is None or dV is None:
        with on(stream):
            dQ, dK, dV = (t if t is not None else torch.empty((n, h, d), dtype=Q.dtype, device=Q.device)
                          for t, n, h in ((dQ, nq, hq), (dK, nk, hkv), (dV, nk, hkv)))
    ws, dt = _ws(workspace, plan, Q, stream), Q.dtype
    _check(_bwd(plan.handle, _code(dt), 1 / math.sqrt(d) if scale is None else scale,
                _view(Q, plan.n_q, hq, d, dt, "Q"), _view(K, plan.n_kv, hkv, d, dt, "K"),
                _view(V, plan.n_kv, hkv, d, dt, "V"), _view(O, plan.n_q, hq, d, dt, "O"),
                None if lse is None else _dense(lse, (hq, plan.n_q), "lse"), _view(dO, nq, hq, d, dt, "dO"),
                _view(dQ, nq, hq, d, dt, "dQ"), _view(dK, nk, hkv, d, dt, "dK"), _view(dV, nk, hkv, d, dt, "dV"),
                ws.data_ptr(), ws.nbytes, _stream_handle(stream)), "dsv_attn_bwd")
    return dQ, dK, dV
