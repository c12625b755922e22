"""What the rotation's calls refuse (CPU only): the binding before the library is called, and the library before any
launch.  Every call here is refused or has nothing to do: nothing is ever launched."""
import ctypes
import types

import pytest
import torch

from paper_2607_28848_amd import dsv, rope
from paper_2607_28848_amd.attn import View

STREAM = types.SimpleNamespace(cuda_stream=0)
N = 6


def args(**changed):
    t = dict(Q=torch.zeros((N, 4, 64)), K=torch.zeros((N, 2, 64)), pos=torch.zeros(N, dtype=torch.int32),
             freq=torch.zeros(16, dtype=torch.float64), q_weight=torch.ones(64), k_weight=torch.ones(64), V=torch.zeros((N, 2, 64)),
             Q_out=torch.zeros((N, 4, 64)), K_out=torch.zeros((N, 2, 64)), V_out=torch.zeros((N, 2, 64)), stream=STREAM)
    t.update(changed)
    return t


def back(**changed):
    t = dict(dQ=torch.zeros((3, 4, 64)), dK=torch.zeros((3, 2, 64)), pos=torch.zeros(N, dtype=torch.int32),
             freq=torch.zeros(16, dtype=torch.float64), rows=torch.zeros(3, dtype=torch.int32), Q=torch.zeros((N, 4, 64)),
             K=torch.zeros((N, 2, 64)), q_weight=torch.ones(64), k_weight=torch.ones(64), dQ_out=torch.zeros((3, 4, 64)),
             dK_out=torch.zeros((3, 2, 64)), dq_weight=torch.zeros(64), dk_weight=torch.zeros(64),
             workspace=torch.zeros(0, dtype=torch.uint8), stream=STREAM)
    t.update(changed)
    return t


def test_the_backward_as_it_is_reaches_the_library():
    with pytest.raises(dsv.DsvError):  # no workspace
        rope.bwd(**back())


@pytest.mark.parametrize("changed", [
    dict(Q=torch.zeros((N, 1, 64)).expand(N, 4, 64)), dict(K=torch.zeros((1, 2, 64)).expand(N, 2, 64)),
    dict(V_out=torch.zeros((1, 2, 64)).expand(N, 2, 64)), dict(Q_out=torch.zeros((N + 1, 4, 64))), dict(V=torch.zeros((N, 3, 64))),
    dict(K_out=torch.zeros((N + 1, 2, 64))), dict(K=torch.zeros((N, 2 * 64))), dict(Q=torch.zeros((N, 4, 128))[..., ::2]),
    dict(pos=torch.zeros(N + 1, dtype=torch.int32)), dict(pos=torch.zeros(2 * N, dtype=torch.int32)[::2]),
    dict(pos=torch.zeros(N, dtype=torch.int64)), dict(pos=None, K=None), dict(freq=torch.zeros(16)),
    dict(q_weight=torch.ones(32)), dict(k_weight=torch.ones(64, dtype=torch.float64)), dict(V=None), dict(K=None),
    dict(slots=torch.zeros(N + 1, dtype=torch.int32)), dict(slots=torch.zeros(N, dtype=torch.int32), V_out=None),
    dict(slots=torch.zeros(N, dtype=torch.int32), K_out=None), dict(Q=None, K=None),
    dict(pos=torch.zeros(N, dtype=torch.int32, device="meta"))])
def test_forward_refuses(changed):
    with pytest.raises(ValueError):
        rope.fwd(**args(**changed))


@pytest.mark.parametrize("changed", [dict(K=torch.zeros((N, 2, 64), dtype=torch.bfloat16)),
                                     dict(Q=torch.zeros((N, 4, 64), dtype=torch.float16))])
def test_types(changed):
    with pytest.raises(TypeError):
        rope.fwd(**args(**changed))


@pytest.mark.parametrize("changed", [
    dict(freq=torch.zeros(36, dtype=torch.float64)), dict(freq=torch.zeros(4, dtype=torch.float64)), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40), dict(eps=1e39),
    dict(Q=torch.zeros((N, 4, 32)), K=None, V=None, K_out=None, V_out=None, Q_out=torch.zeros((N, 4, 32)), q_weight=None),
    dict(Q=torch.zeros((N, 4, 66))[..., :64]), dict(Q=torch.zeros(4 * N * 64 + 1)[1:].view(N, 4, 64)),
    dict(Q_out=torch.zeros(N * 64 + 1024).as_strided((N, 4, 64), (64, 64, 1)))])
def test_library_refuses(changed):
    with pytest.raises(dsv.DsvError):
        rope.fwd(**args(**changed))


@pytest.mark.parametrize("changed", [
    dict(Q=None), dict(K=None), dict(q_weight=None), dict(dK=None, dk_weight=torch.zeros(64)), dict(dQ=None, dK=None),
    dict(rows=torch.zeros(4, dtype=torch.int32)), dict(dQ_out=torch.zeros((2, 4, 64))), dict(dK=torch.zeros((1, 2, 64)).expand(3, 2, 64)),
    dict(dq_weight=torch.zeros(32)), dict(rows=torch.zeros(3, dtype=torch.int32, device="meta"))])
def test_backward_refuses(changed):
    with pytest.raises(ValueError):
        rope.bwd(**back(**changed))


def test_more_gradient_rows_than_rows():
    with pytest.raises(dsv.DsvError):
        rope.bwd(**back(rows=None, dQ=torch.zeros((N + 1, 4, 64)), dK=torch.zeros((N + 1, 2, 64)), dQ_out=torch.zeros((N + 1, 4, 64)),
                        dK_out=torch.zeros((N + 1, 2, 64)), dq_weight=None, dk_weight=None))


def test_c_entries():
    """Null pointers and counts, straight through the library."""
    fwd, bwd = rope._lib.dsv_rope_fwd, rope._lib.dsv_rope_bwd
    x = torch.zeros(64 * 8 * N)
    f = torch.zeros(32, dtype=torch.float64)
    p = torch.zeros(N, dtype=torch.int32)
    v = View(x.data_ptr(), 0, 0)
    r = ctypes.byref

    def base(**c):
        s = rope.Rope(N, 2, 1, 64, 64, 0, 1e-6, p.data_ptr(), f.data_ptr(), None, None)
        for k, value in c.items():
            setattr(s, k, value)
        return s

    def call(s, Q=v, K=v, V=v, Qo=v, Ko=v, Vo=v, dt=1, slots=None, n_slots=0):
        o = [None if t is None else r(t) for t in (Q, K, V, Qo, Ko, Vo)]
        return fwd(dt, None if s is None else r(s), o[0], o[1], o[2], slots, n_slots, o[3], o[4], o[5], None)

    none = View(None, 0, 0)
    for s, kw in ((None, {}), (base(n=-1), {}), (base(pos=None), {}), (base(freq=None), {}), (base(), dict(Q=None)),
                  (base(), dict(Ko=None)), (base(), dict(V=None)), (base(), dict(Vo=None)), (base(), dict(Q=none)),
                  (base(), dict(slots=p.data_ptr(), n_slots=-1)), (base(), dict(slots=p.data_ptr() + 1, n_slots=1)),
                  (base(freq=f.data_ptr() + 4), {}), (base(q_weight=f.data_ptr() + 8), {})):
        assert call(s, **kw) == -1, kw
    for s, kw in ((base(heads_q=-1), {}), (base(heads_q=0, heads_kv=0), {}), (base(heads_q=1025), {}), (base(head_dim=96), {}),
                  (base(rotated=8), {}), (base(rotated=80), {}), (base(interleaved=2), {}), (base(), dict(dt=2))):
        assert call(s, **kw) == -2, kw
    for kw in (dict(Q=View(x.data_ptr(), 60, 64)), dict(Q=View(x.data_ptr(), 1 << 24, 64)), dict(Ko=View(x.data_ptr(), 132, 64))):
        assert call(base(), **kw) == -4, kw
    assert call(base(n=0)) == 0
    assert call(base(n=0, pos=None), Q=none, K=none, V=none, Qo=none, Ko=none, Vo=none) == 0

    def go_back(s, m=2, rows=p.data_ptr(), dQ=v, dK=v, Q=v, K=v, dqw=None, dkw=None, ws=None, bytes=0):
        return bwd(1, r(s), m, rows, r(dQ), r(dK), None if Q is None else r(Q), None if K is None else r(K), r(dQ), r(dK), dqw, dkw, ws,
                   bytes, None)
    w = torch.ones(64)
    normed = base(q_weight=w.data_ptr(), k_weight=w.data_ptr())
    assert go_back(base(), m=-1) == -1 and go_back(base(), m=N + 1, rows=None) == -1
    assert go_back(base(), dqw=w.data_ptr()) == -1 and go_back(normed, Q=None) == -1
    assert go_back(normed, dqw=w.data_ptr()) == -1  # no workspace
    room = torch.zeros(1024, dtype=torch.float64)
    at = (room.data_ptr() + 255) & ~255
    assert go_back(normed, dqw=w.data_ptr(), ws=at, bytes=64) == -4 and go_back(normed, dkw=w.data_ptr(), ws=at + 8, bytes=4096) == -1
    assert go_back(base(), m=0) == 0
    n = ctypes.c_size_t(0)
    assert rope._lib.dsv_rope_workspace(r(base()), -1, r(n)) == -1 and rope._lib.dsv_rope_workspace(r(base()), 5, None) == -1
    assert rope._lib.dsv_rope_workspace(r(base(head_dim=32)), 5, r(n)) == -2


def test_workspace_grows_to_its_end():
    sizes = [rope.workspace_bytes(m, 32, 8, 128) for m in (0, 1, 7, 100, 5000, 1 << 20, (1 << 31) - 1)]
    assert sizes == sorted(sizes) and sizes[0] >= 256 and sizes[-1] == sizes[-2]
    with pytest.raises(ValueError):
        rope.workspace_bytes(1 << 31, 32, 8, 128)
