"""Binding of the norms and the position rotation (dsv_rope_* of include/dsv.h): argument marshalling only.

    freq = rope.frequencies(128, 500000.0, device="cuda")
    Q, K, V = rope.fwd(q, k, pos, freq, q_weight=wq, k_weight=wk, V=v, K_out=cache_k, V_out=cache_v, slots=slots)
    dq, dk, dwq, dwk = rope.bwd(dQ, dK, pos, freq, rows=train_rows, Q=q, K=k, q_weight=wq, k_weight=wk)

q, k and v are the columns of the q/k/v product's rows, [n][heads][d]; pos [n] int32; K and V go to the rows of a cache
that slots [n] int32 name (without slots, row i to row i).  The backward serves the fine-tuning rows in compact order:
gradient row i belongs to row rows[i] of the batch.  Tensors may be any views whose head vectors are contiguous, but not
broadcast ones; outputs may be the inputs themselves.
"""
from __future__ import annotations

import ctypes
import struct

from . import dsv
from .attn import View, _code, _marshal, _view, here, int32, launchable, made
from .dsv import OK, _check, _stream_handle, torch

_lib = dsv.lib_handle()
_vp, _i32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t


class Rope(ctypes.Structure):
    _fields_ = [("n", _i32), ("heads_q", _i32), ("heads_kv", _i32), ("head_dim", _i32), ("rotated", _i32),
                ("interleaved", _i32), ("eps", ctypes.c_double), ("pos", _vp), ("freq", _vp), ("q_weight", _vp),
                ("k_weight", _vp)]


_ropep = ctypes.POINTER(Rope)
_viewp = ctypes.POINTER(View)
_lib.dsv_rope_workspace.argtypes = [_ropep, _i32, ctypes.POINTER(_sz)]
_lib.dsv_rope_workspace.restype = ctypes.c_int
_lib.dsv_rope_fwd.argtypes = [ctypes.c_int, _ropep] + [_viewp] * 3 + [_vp, _i32] + [_viewp] * 3 + [_vp]
_lib.dsv_rope_fwd.restype = ctypes.c_int
_lib.dsv_rope_bwd.argtypes = [ctypes.c_int, _ropep, _i32, _vp] + [_viewp] * 6 + [_vp, _vp, _vp, _sz, _vp]
_lib.dsv_rope_bwd.restype = ctypes.c_int

# The calls below pass their structures as packed bytes, read during the call only, as the attention's do: the rotation of
# a decode step takes the GPU 3 us, and marshalling structures takes the host several times that.
_fwd = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_int, *[_vp] * 5, _i32, *[_vp] * 4)(("dsv_rope_fwd", _lib))
_bwd = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_int, _vp, _i32, *[_vp] * 10, _sz, _vp)(("dsv_rope_bwd", _lib))
_ROPE_PACK = struct.Struct("@6id4P").pack
assert len(_ROPE_PACK(*[0] * 6, 0.0, *[0] * 4)) == ctypes.sizeof(Rope)


def frequencies(rotated: int, theta: float = 10000.0, device=None):
    """freq [rotated / 2], radians a position: theta^(-2 i / rotated)."""
    return theta ** (-torch.arange(0, rotated, 2, dtype=torch.float64, device=device) / max(rotated, 1))


_vec = _marshal.vec  # (t, n, dtype, name): the address of a vector, 0 for None


def _heads(t, name: str):
    if t.dim() != 3:
        raise ValueError("%s must be [rows][heads][head_dim], got %s" % (name, tuple(t.shape)))
    return t.shape


def _rope(n, hq, hkv, d, pos, freq, q_weight, k_weight, eps, interleaved) -> bytes:
    rotated = 0 if freq is None else 2 * freq.shape[0]
    if n >= 1 << 31 or max(hq, hkv, d, rotated) >= 1 << 31:
        int32(n=n, heads_q=hq, heads_kv=hkv, head_dim=d, rotated=rotated)
    return _ROPE_PACK(n, hq, hkv, d, rotated, 1 if interleaved else 0, eps,
                      0 if freq is None else _vec(pos, n, torch.int32, "pos"), _vec(freq, rotated // 2, torch.float64, "freq"),
                      _vec(q_weight, d, torch.float32, "q_weight"), _vec(k_weight, d, torch.float32, "k_weight"))


def workspace_bytes(n_rows: int, heads_q: int, heads_kv: int, head_dim: int) -> int:
    """Bytes of device workspace for the weights' gradients over n_rows gradient rows."""
    n = _sz(0)
    n_rows, heads_q, heads_kv, head_dim = int32(n_rows=n_rows, heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim)
    _check(_lib.dsv_rope_workspace(ctypes.byref(Rope(0, heads_q, heads_kv, head_dim)), n_rows, ctypes.byref(n)),
           "dsv_rope_workspace")
    return int(n.value)


def fwd(Q, K, pos, freq, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, V=None, slots=None, Q_out=None,
        K_out=None, V_out=None, stream=None):
    """dsv_rope_fwd; returns (Q_out, K_out), or (Q_out, K_out, V_out) given V.  Q or K None: keys or queries alone.  freq
    None: no rotation (pos may be None).  K_out and V_out are needed with slots; what is not given else is made."""
    if Q is None and K is None:
        raise ValueError("neither Q nor K")
    if K is None and not (V is None and slots is None and K_out is None and V_out is None):
        raise ValueError("V, slots, K_out and V_out need K")
    if V is None and V_out is not None:
        raise ValueError("V_out needs V")
    like = K if Q is None else Q
    n, _, d = _heads(like, "Q" if Q is not None else "K")
    hq, hkv, dt = 0 if Q is None else Q.shape[1], 0 if K is None else _heads(K, "K")[1], like.dtype
    if slots is not None and (K_out is None or (V is not None and V_out is None)):
        raise ValueError("slots need K_out, and V_out where V is given")
    host = here(Q, K, V, pos, freq, q_weight, k_weight, slots, Q_out, K_out, V_out, stream=stream)
    if hq:
        Q_out = made(Q_out, (n, hq, d), dt, Q, stream)
    if hkv:
        K_out = made(K_out, (n, hkv, d), dt, K, stream)
    if V is not None:
        V_out = made(V_out, (n, hkv, d), dt, V, stream)
    rows = n if slots is None else K_out.shape[0]
    if rows >= 1 << 31:
        int32(n_slots=rows)
    r = _rope(n, hq, hkv, d, pos, freq, q_weight if hq else None, k_weight if hkv else None, eps, interleaved)
    args = (_code(dt), r, None if Q is None else _view(Q, n, hq, d, dt, "Q"),
            None if K is None else _view(K, n, hkv, d, dt, "K"), None if V is None else _view(V, n, hkv, d, dt, "V"),
            None if slots is None else _vec(slots, n, torch.int32, "slots"), rows,
            None if Q is None else _view(Q_out, n, hq, d, dt, "Q_out"),
            None if K is None else _view(K_out, rows, hkv, d, dt, "K_out"),
            None if V is None else _view(V_out, rows, hkv, d, dt, "V_out"))
    if host:
        launchable(host, n > 0, "rope.fwd")
    rc = _fwd(*args, _stream_handle(stream))
    if rc != OK:
        _check(rc, "dsv_rope_fwd")
    return (Q_out, K_out) if V is None else (Q_out, K_out, V_out)


def bwd(dQ, dK, pos, freq, rows=None, Q=None, K=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
        dQ_out=None, dK_out=None, dq_weight=None, dk_weight=None, want_weights=None, workspace=None, stream=None):
    """dsv_rope_bwd; returns (dQ_out, dK_out, dq_weight, dk_weight).  Q, K: the forward's inputs, needed where there is a
    weight; they or pos state the batch's rows, outside which a gradient row gets zeros (none given: any row from 0 on is one).  The weights' gradients are fp32 and overwritten; one not given is made if want_weights, which stands for
    "where its gradient's rows are made" if None, else it is not computed and None is returned for it."""
    if dQ is None and dK is None:
        raise ValueError("neither dQ nor dK")
    if (dQ is not None and q_weight is not None and Q is None) or (dK is not None and k_weight is not None and K is None):
        raise ValueError("the norm's gradient needs the forward's Q and K")
    like = dK if dQ is None else dQ
    m, _, d = _heads(like, "dQ" if dQ is not None else "dK")
    hq, hkv, dt = 0 if dQ is None else dQ.shape[1], 0 if dK is None else _heads(dK, "dK")[1], like.dtype
    if (dQ is None or q_weight is None) and dq_weight is not None or (dK is None or k_weight is None) and dk_weight is not None:
        raise ValueError("the gradient of a weight that is not there")
    stated = next((t for t in (pos, Q, K) if t is not None), None)
    # nothing of a batch's rows is read where nothing states their number: every row that 32 bits name is one
    n = stated.shape[0] if stated is not None else m if rows is None else (1 << 31) - 1
    host = here(dQ, dK, pos, freq, rows, Q, K, q_weight, k_weight, dQ_out, dK_out, dq_weight, dk_weight, workspace,
                stream=stream)
    if hq and q_weight is not None and (dQ_out is None if want_weights is None else want_weights):
        dq_weight = made(dq_weight, (d,), torch.float32, dQ, stream)
    if hkv and k_weight is not None and (dK_out is None if want_weights is None else want_weights):
        dk_weight = made(dk_weight, (d,), torch.float32, dK, stream)
    if hq:
        dQ_out = made(dQ_out, (m, hq, d), dt, dQ, stream)
    if hkv:
        dK_out = made(dK_out, (m, hkv, d), dt, dK, stream)
    if workspace is None and not (dq_weight is None and dk_weight is None):
        workspace = made(None, (workspace_bytes(m, hq, hkv, d),), torch.uint8, like, stream)
    r = _rope(n, hq, hkv, d, pos, freq, q_weight if hq else None, k_weight if hkv else None, eps, interleaved)

    def view(t, rows, heads, name):
        return None if t is None else _view(t, rows, heads, d, dt, name)

    if m >= 1 << 31:
        int32(n_rows=m)
    args = (_code(dt), r, m, None if rows is None else _vec(rows, m, torch.int32, "rows"), view(dQ, m, hq, "dQ"),
            view(dK, m, hkv, "dK"), view(Q, n, hq, "Q") if hq and q_weight is not None else None,
            view(K, n, hkv, "K") if hkv and k_weight is not None else None, view(dQ_out, m, hq, "dQ_out") if hq else None,
            view(dK_out, m, hkv, "dK_out") if hkv else None, _vec(dq_weight, d, torch.float32, "dq_weight"),
            _vec(dk_weight, d, torch.float32, "dk_weight"), None if workspace is None else workspace.data_ptr(),
            0 if workspace is None else workspace.nbytes)
    if host:
        launchable(host, m > 0 or dq_weight is not None or dk_weight is not None, "rope.bwd")
    rc = _bwd(*args, _stream_handle(stream))
    if rc != OK:
        _check(rc, "dsv_rope_bwd")
    return dQ_out if hq else None, dK_out if hkv else None, dq_weight, dk_weight
