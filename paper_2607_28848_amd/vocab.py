"""Binding of the vocabulary loss (dsv_vocab_* of include/dsv.h): argument marshalling only.

    losses = vocab.loss(X, W, target)                              # scoring
    losses, dX = vocab.loss_grad(X, W, target, weight=weight)      # the start of a fine-tuning step's backward
    losses = vocab.distill(X, W, ids, teacher, temperature=2.0)    # against a teacher's top logits
    losses, dX = vocab.distill_grad(X, W, ids, teacher, temperature=2.0, weight=weight)

X [T][K] are the rows' last hidden states, W [V][K] the head, target [T] int32 (outside [0, V): a row without one).
ids [T][k] int32 and teacher [T][k] fp32 are a teacher's k largest logits a row (an id outside [0, V): padding).
"""
from __future__ import annotations

import ctypes

from . import dsv
from .attn import here, int32, launchable, on
from .dsv import _check, _ptr, _stream_handle, torch

_lib = dsv.lib_handle()
_vp, _i32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_lib.dsv_vocab_workspace.argtypes = [ctypes.c_int, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(_sz)]
_lib.dsv_vocab_workspace.restype = ctypes.c_int
_lib.dsv_vocab_loss.argtypes = [ctypes.c_int, _i32, _i32, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]
_lib.dsv_vocab_loss.restype = ctypes.c_int
_lib.dsv_vocab_loss_grad.argtypes = ([ctypes.c_int, _i32, _i32, _i32, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _vp,
                                      _i32, _vp, _sz, _vp])
_lib.dsv_vocab_loss_grad.restype = ctypes.c_int

_lib.dsv_vocab_distill_workspace.argtypes = [ctypes.c_int] + [_i32] * 6 + [ctypes.POINTER(_sz)]
_lib.dsv_vocab_distill_workspace.restype = ctypes.c_int
_lib.dsv_vocab_distill.argtypes = ([ctypes.c_int] + [_i32] * 4 + [_vp, _i32, _vp, _i32, _vp, _vp, ctypes.c_double, _vp, _vp, _sz,
                                                                  _vp])
_lib.dsv_vocab_distill.restype = ctypes.c_int
_lib.dsv_vocab_distill_grad.argtypes = ([ctypes.c_int] + [_i32] * 4 + [_vp, _i32, _vp, _i32, _vp, _i32, _vp, _vp, ctypes.c_double,
                                                                       _vp, _vp, _vp, _i32, _vp, _sz, _vp])
_lib.dsv_vocab_distill_grad.restype = ctypes.c_int


def _code(dtype) -> int:
    if dtype == torch.bfloat16:
        return dsv.BF16
    if dtype == torch.float32:
        return dsv.F32
    raise TypeError("dsv supports bfloat16 and float32 tensors, got %s" % dtype)


def workspace_bytes(T: int, K: int, V: int, dtype, grad: bool, ldw: int = 0) -> int:
    """Bytes of device workspace; ldw: the head's row stride where it is not dense."""
    n = _sz(0)
    T, K, V, ldw = int32(T=T, K=K, V=V, ldw=ldw)
    _check(_lib.dsv_vocab_workspace(_code(dtype), T, K, V, ldw, 1 if grad else 0, ctypes.byref(n)), "dsv_vocab_workspace")
    return int(n.value)


def _mat(t, rows: int, cols: int, dtype, name: str):
    """(address, row stride: 0 when dense) of a matrix with contiguous rows."""
    if t.dtype != dtype:
        raise TypeError("%s is %s, the call's tensors are %s" % (name, t.dtype, dtype))
    if tuple(t.shape) != (rows, cols):
        raise ValueError("%s must be [%d][%d], got %s" % (name, rows, cols, tuple(t.shape)))
    if t.numel() and cols > 1 and t.stride(1) != 1:
        raise ValueError("%s: the elements of a row must be contiguous" % name)
    if rows > 1 and t.stride(0) == 0:  # the library takes 0 for the dense stride
        raise ValueError("%s is broadcast (a row stride of 0): make it contiguous" % name)
    ld = 0 if rows <= 1 or t.stride(0) == cols else t.stride(0)
    if max(rows, cols, ld) >= 1 << 31:  # the library takes 32 bits of them
        raise ValueError("%s: [%d][%d] of row stride %d does not fit 32 bits" % (name, rows, cols, ld))
    return t.data_ptr(), ld


def _vec(t, n: int, dtype, name: str):
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != (n,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements" % (name, dtype, n))
    return t.data_ptr()


def _ws(given, like, T, K, V, grad, ldw, stream):
    if given is None:
        with on(stream):
            given = torch.empty(workspace_bytes(T, K, V, like.dtype, grad, ldw), dtype=torch.uint8, device=like.device)
    return given, given.numel() * given.element_size()


def _new(given, shape, dtype, device, stream):
    if given is not None:
        return given
    with on(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def loss(X, W, target, loss=None, workspace=None, stream=None):
    """dsv_vocab_loss: -log softmax(X W^T)[target] of every row, fp32."""
    (T, K), V = X.shape, W.shape[0]
    host = here(X, W, target, loss, workspace, stream=stream)
    loss = _new(loss, (T,), torch.float32, X.device, stream)
    (x, ldx), (w, ldw) = _mat(X, T, K, X.dtype, "X"), _mat(W, V, K, X.dtype, "W")
    ws, n = _ws(workspace, X, T, K, V, False, ldw, stream)
    launchable(host, T > 0, "vocab.loss")
    _check(_lib.dsv_vocab_loss(_code(X.dtype), T, K, V, x, ldx, w, ldw, _vec(target, T, torch.int32, "target"),
                               _vec(loss, T, torch.float32, "loss"), _ptr(ws), n, _stream_handle(stream)),
           "dsv_vocab_loss")
    return loss


def loss_grad(X, W, target, weight=None, Wt=None, loss=None, dX=None, workspace=None, stream=None):
    """dsv_vocab_loss_grad; returns (loss, dX).  weight [T] fp32: the upstream gradient of each row's loss (ones if
    None).  Wt [K][V]: the head transposed, kept by the caller (read for bf16 where V is a multiple of 8 below 2^22)."""
    (T, K), V = X.shape, W.shape[0]
    host = here(X, W, target, weight, Wt, loss, dX, workspace, stream=stream)
    loss = _new(loss, (T,), torch.float32, X.device, stream)
    dX = _new(dX, (T, K), X.dtype, X.device, stream)
    (x, ldx), (w, ldw), (dx, lddx) = _mat(X, T, K, X.dtype, "X"), _mat(W, V, K, X.dtype, "W"), _mat(dX, T, K, X.dtype, "dX")
    wt, ldwt = _mat(Wt, K, V, X.dtype, "Wt") if Wt is not None else (None, 0)
    ws, n = _ws(workspace, X, T, K, V, True, ldw, stream)
    launchable(host, T > 0, "vocab.loss_grad")
    _check(_lib.dsv_vocab_loss_grad(_code(X.dtype), T, K, V, x, ldx, w, ldw, wt, ldwt,
                                    _vec(target, T, torch.int32, "target"), _vec(weight, T, torch.float32, "weight"),
                                    _vec(loss, T, torch.float32, "loss"), dx, lddx, _ptr(ws), n, _stream_handle(stream)),
           "dsv_vocab_loss_grad")
    return loss, dX


def distill_workspace_bytes(T: int, K: int, V: int, k: int, dtype, grad: bool, ldw: int = 0) -> int:
    """Bytes of device workspace; ldw: the head's row stride where it is not dense."""
    n = _sz(0)
    T, K, V, k, ldw = int32(T=T, K=K, V=V, k=k, ldw=ldw)
    _check(_lib.dsv_vocab_distill_workspace(_code(dtype), T, K, V, k, ldw, 1 if grad else 0, ctypes.byref(n)),
           "dsv_vocab_distill_workspace")
    return int(n.value)


def _entries(t, T: int, k: int, dtype, name: str):
    if t.dtype != dtype or tuple(t.shape) != (T, k) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape [%d][%d]" % (name, dtype, T, k))
    return t.data_ptr()


def _distill_ws(given, like, T, K, V, k, grad, ldw, stream):
    if given is None:
        n = distill_workspace_bytes(T, K, V, k, like.dtype, grad, ldw)
        with on(stream):
            given = torch.empty(n, dtype=torch.uint8, device=like.device)
    return given, given.numel() * given.element_size()


def distill(X, W, ids, teacher, temperature=1.0, loss=None, workspace=None, stream=None):
    """dsv_vocab_distill: the divergence of softmax(X W^T / temperature) from the teacher of every row, fp32."""
    (T, K), V, k = X.shape, W.shape[0], ids.shape[-1]
    host = here(X, W, ids, teacher, loss, workspace, stream=stream)
    loss = _new(loss, (T,), torch.float32, X.device, stream)
    (x, ldx), (w, ldw) = _mat(X, T, K, X.dtype, "X"), _mat(W, V, K, X.dtype, "W")
    i, t = _entries(ids, T, k, torch.int32, "ids"), _entries(teacher, T, k, torch.float32, "teacher")
    ws, n = _distill_ws(workspace, X, T, K, V, k, False, ldw, stream)
    launchable(host, T > 0, "vocab.distill")
    _check(_lib.dsv_vocab_distill(_code(X.dtype), T, K, V, k, x, ldx, w, ldw, i, t, temperature,
                                  _vec(loss, T, torch.float32, "loss"), _ptr(ws), n, _stream_handle(stream)),
           "dsv_vocab_distill")
    return loss


def distill_grad(X, W, ids, teacher, temperature=1.0, weight=None, Wt=None, loss=None, dX=None, workspace=None, stream=None):
    """dsv_vocab_distill_grad; returns (loss, dX).  weight [T] fp32: the upstream gradient of each row's loss (ones if
    None).  Wt [K][V]: the head transposed, as loss_grad takes it."""
    (T, K), V, k = X.shape, W.shape[0], ids.shape[-1]
    host = here(X, W, ids, teacher, weight, Wt, loss, dX, workspace, stream=stream)
    loss = _new(loss, (T,), torch.float32, X.device, stream)
    dX = _new(dX, (T, K), X.dtype, X.device, stream)
    (x, ldx), (w, ldw), (dx, lddx) = _mat(X, T, K, X.dtype, "X"), _mat(W, V, K, X.dtype, "W"), _mat(dX, T, K, X.dtype, "dX")
    wt, ldwt = _mat(Wt, K, V, X.dtype, "Wt") if Wt is not None else (None, 0)
    i, t = _entries(ids, T, k, torch.int32, "ids"), _entries(teacher, T, k, torch.float32, "teacher")
    ws, n = _distill_ws(workspace, X, T, K, V, k, True, ldw, stream)
    launchable(host, T > 0, "vocab.distill_grad")
    _check(_lib.dsv_vocab_distill_grad(_code(X.dtype), T, K, V, k, x, ldx, w, ldw, wt, ldwt, i, t, temperature,
                                       _vec(weight, T, torch.float32, "weight"), _vec(loss, T, torch.float32, "loss"), dx, lddx,
                                       _ptr(ws), n, _stream_handle(stream)), "dsv_vocab_distill_grad")
    return loss, dX
