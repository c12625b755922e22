"""Plans with a window on the host: what is refused, and that no more is laid down than the window needs (CPU only)."""
import ctypes

import numpy as np
import pytest

from paper_2607_28848_amd import attn, dsv

lib = dsv.lib_handle()


def build(window, sinks, seqs=((0, 10, 0, 10, 0),), nq=100, nk=100, hq=8, hkv=2, d=128):
    s = np.ascontiguousarray(np.asarray(seqs, np.int32).reshape(-1, 5))
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    rc = lib.dsv_attn_build_window(s.ctypes.data, s.shape[0], nq, nk, hq, hkv, d, window, sinks, ctypes.byref(n), ctypes.byref(h))
    if h.value:
        lib.dsv_attn_free(h)
    return rc


@pytest.mark.parametrize("window,sinks,want", [(1, 0, dsv.OK), (0, 0, dsv.ERR_RANGE), (-5, 0, dsv.ERR_RANGE), (3, -1, dsv.ERR_RANGE),
                                               (2 ** 31 - 1, 2 ** 31 - 1, dsv.OK), (1, 2 ** 31 - 1, dsv.OK)])
def test_build(window, sinks, want):
    assert build(window, sinks) == want


@pytest.mark.parametrize("seqs", [[(0, 10, 0, 10, 2)], [(95, 10, 0, 10, 0)], [(0, 10, 95, 10, 0)], [(20, 10, 0, 10, 0), (0, 21, 0, 10, 0)]])
def test_build_refuses_what_the_plain_plan_refuses(seqs):
    assert build(5, 1, seqs) in (dsv.ERR_RANGE, dsv.ERR_LAYOUT)


def test_build_refuses_null():
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    assert lib.dsv_attn_build_window(None, 1, 10, 10, 2, 2, 64, 5, 0, ctypes.byref(n), ctypes.byref(h)) == dsv.ERR_ARG
    assert lib.dsv_attn_build_window(None, 0, 10, 10, 2, 2, 64, 5, 0, None, ctypes.byref(h)) == dsv.ERR_ARG
    assert lib.dsv_attn_build_window(None, 0, 10, 10, 2, 2, 64, 5, 0, ctypes.byref(n), None) == dsv.ERR_ARG


def test_binding():
    seqs = [(0, 10, 0, 10, 0)]
    with pytest.raises(ValueError):
        attn.Plan(seqs, 10, 10, 4, 2, 64, sinks=3)
    for w in (1 << 31, -(1 << 31) - 1):
        with pytest.raises(ValueError):
            attn.Plan(seqs, 10, 10, 4, 2, 64, window=w)
    with pytest.raises(ValueError):
        attn.Plan(seqs, 10, 10, 4, 2, 64, window=4, sinks=1 << 31)
    for w, s in ((0, 0), (4, -1)):
        with pytest.raises(dsv.DsvError):
            attn.Plan(seqs, 10, 10, 4, 2, 64, window=w, sinks=s)
    p = attn.Plan(seqs, 10, 10, 4, 2, 64, window=4, sinks=1)
    assert (p.window, p.sinks) == (4, 1)


def test_a_decode_token_costs_its_window():
    """Pieces (and their sums' room) follow the window, not the cache."""
    seqs = [(i, 1, 0, 1000000, 0) for i in range(4)]
    plain = attn.Plan(seqs, 4, 1000000, 8, 2, 128)
    some = attn.Plan(seqs, 4, 1000000, 8, 2, 128, window=500, sinks=4)
    short = attn.Plan([(i, 1, 0, 504, 0) for i in range(4)], 4, 1000000, 8, 2, 128)
    bf = attn.torch.bfloat16
    assert attn.workspace_bytes(some, bf) == attn.workspace_bytes(short, bf) < attn.workspace_bytes(plain, bf)


def test_the_widest_numbers():
    """Sequences, windows and sinks at the ends of 32 bits: sums of them do not wrap."""
    m = 2 ** 31 - 1
    for k in (m, m - 1024):
        for w, s, q in ((1, 0, 1), (m, m, 40), (k - 1, 0, 40), (k - 1, 0, 1), (1, k - 2, 40), (1, k - 2, 1), (1000, 1000, 40),
                        (1, m, 1), (k - 33, 33, 1)):
            hides = k > w and s < k - w
            try:
                p = attn.Plan([(0, 2, 0, 100000, 1), (2, q, 0, k, 0)], 43, m, 1, 1, 64, window=w, sinks=s)
            except dsv.DsvError as e:
                assert hides and k == m and e.status == dsv.ERR_SIZE
            else:
                assert (not hides or k < m) and attn.workspace_bytes(p, attn.torch.bfloat16) > 0
                del p
