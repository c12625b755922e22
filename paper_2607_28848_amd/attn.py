"""Binding of the attention calls (dsv_attn_* of include/dsv.h): argument marshalling only.

One plan holds a mixed batch's sequences -- whole prompts, chunks behind a cached prefix, single decode tokens and
fine-tuning samples -- and serves every layer:

    plan = attn.Plan([(q_start, q_len, k_start, k_len, is_train), ...], n_q, n_kv, heads_q, heads_kv, head_dim,
                     device="cuda")
    O, lse = attn.fwd(plan, Q, K, V)                      # Q [n_q][heads_q][d]; K, V [n_kv][heads_kv][d]
    dQ, dK, dV = attn.bwd(plan, Q, K, V, O, lse, dO)      # rows of the fine-tuning samples alone ("compact order")

Query i of a sequence sees its keys j <= i + k_len - q_len.  Tensors may be any views whose head vectors are
contiguous: columns of a q/k/v product, a cache laid out [row][head][d] or [head][row][d].
"""
from __future__ import annotations

import ctypes
import math

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


class Plan:
    """The packed sequences of a batch.  device=None builds a host-only plan (inspection only)."""

    def __init__(self, seqs, n_q: int, n_kv: int, heads_q: int, heads_kv: int, head_dim: int, device=None, stream=None):
        self.seqs = np.ascontiguousarray(np.asarray(seqs, np.int32).reshape(-1, 5))
        self.n_q, self.n_kv = int(n_q), int(n_kv)
        self.heads_q, self.heads_kv, self.head_dim = int(heads_q), int(heads_kv), int(head_dim)
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


def _view(t, rows: int, heads: int, d: int, dtype, name: str):
    if t.dtype != dtype:
        raise TypeError("%s is %s, the call's tensors are %s" % (name, t.dtype, dtype))
    if t.dim() == 2 and t.shape[1] == heads * d:
        t = t.unflatten(1, (heads, d))
    if tuple(t.shape) != (rows, heads, d):
        raise ValueError("%s must be [%d][%d][%d], got %s" % (name, rows, heads, d, tuple(t.shape)))
    if t.numel() and t.stride(2) != 1:
        raise ValueError("%s: the elements of a head must be contiguous" % name)
    # a stride of a dimension of one is arbitrary: the dense one then
    return View(t.data_ptr(), t.stride(0) if rows > 1 else 0, t.stride(1) if heads > 1 and rows > 0 else 0)


def _dense(t, shape, name: str):
    if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError("%s must be a contiguous fp32 tensor of shape %s" % (name, shape))
    return t.data_ptr()


def _ws(given, plan, like):
    return given if given is not None else torch.empty(workspace_bytes(plan, like.dtype), dtype=torch.uint8,
                                                       device=like.device)


def fwd(plan: Plan, Q, K, V, scale=None, O=None, lse=None, want_lse: bool = True, workspace=None, stream=None):
    """dsv_attn_fwd; returns (O, lse).  scale: 1 / sqrt(head_dim) if None.  lse is [heads_q][n_q] fp32; with
    want_lse=False and no lse given none is written (inference)."""
    hq, hkv, d = plan.heads_q, plan.heads_kv, plan.head_dim
    made = O is None
    if made:
        # rows that no sequence holds are not written
        O = torch.zeros((plan.n_q, hq, d), dtype=Q.dtype, device=Q.device)
    if lse is None and want_lse and made:
        lse = torch.full((hq, plan.n_q), -math.inf, dtype=torch.float32, device=Q.device)
    ws = _ws(workspace, plan, Q)
    v = [_view(t, n, h, d, Q.dtype, name) for t, n, h, name in ((Q, plan.n_q, hq, "Q"), (K, plan.n_kv, hkv, "K"),
                                                               (V, plan.n_kv, hkv, "V"), (O, plan.n_q, hq, "O"))]
    _check(_lib.dsv_attn_fwd(plan.handle, _code(Q.dtype), 1 / math.sqrt(d) if scale is None else scale, *v,
                             None if lse is None else _dense(lse, (hq, plan.n_q), "lse"), _ptr(ws),
                             ws.numel() * ws.element_size(), _stream_handle(stream)), "dsv_attn_fwd")
    return O, lse


def bwd(plan: Plan, Q, K, V, O, lse, dO, scale=None, dQ=None, dK=None, dV=None, workspace=None, stream=None):
    """dsv_attn_bwd; returns (dQ, dK, dV): [train_q][heads_q][d] and twice [train_k][heads_kv][d]."""
    hq, hkv, d, nq, nk = plan.heads_q, plan.heads_kv, plan.head_dim, plan.train_q, plan.train_k
    dQ, dK, dV = (t if t is not None else torch.empty((n, h, d), dtype=Q.dtype, device=Q.device)
                  for t, n, h in ((dQ, nq, hq), (dK, nk, hkv), (dV, nk, hkv)))
    ws = _ws(workspace, plan, Q)
    v = [_view(t, n, h, d, Q.dtype, name) for t, n, h, name in (
        (Q, plan.n_q, hq, "Q"), (K, plan.n_kv, hkv, "K"), (V, plan.n_kv, hkv, "V"), (O, plan.n_q, hq, "O"),
        (dO, nq, hq, "dO"), (dQ, nq, hq, "dQ"), (dK, nk, hkv, "dK"), (dV, nk, hkv, "dV"))]
    _check(_lib.dsv_attn_bwd(plan.handle, _code(Q.dtype), 1 / math.sqrt(d) if scale is None else scale, *v[:4],
                             _dense(lse, (hq, plan.n_q), "lse"), *v[4:], _ptr(ws), ws.numel() * ws.element_size(),
                             _stream_handle(stream)), "dsv_attn_bwd")
    return dQ, dK, dV
