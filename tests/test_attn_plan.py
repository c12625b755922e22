"""Attention plans and argument checks on the host (no device is needed, nothing is launched)."""
import ctypes

import numpy as np
import pytest

from paper_2607_28848_amd import attn, dsv

lib = dsv.lib_handle()


def build(seqs, nq=100, nk=100, hq=8, hkv=2, d=128):
    s = np.ascontiguousarray(np.asarray(seqs, np.int32).reshape(-1, 5))
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    rc = lib.dsv_attn_build(s.ctypes.data, s.shape[0], nq, nk, hq, hkv, d, ctypes.byref(n), ctypes.byref(h))
    if h.value:
        lib.dsv_attn_free(h)
    return rc


@pytest.mark.parametrize("seqs,kw,want", [
    ([(0, 10, 0, 10, 0)], {}, dsv.OK),
    ([], {}, dsv.OK),
    ([(0, 0, 0, 0, 1)], dict(nq=0, nk=0), dsv.OK),
    ([(0, 10, 0, 10, 2)], {}, dsv.ERR_RANGE),
    ([(0, 10, 0, 10, 0)], dict(hq=0), dsv.ERR_RANGE),
    ([(0, 10, 0, 10, 0)], dict(hkv=0), dsv.ERR_RANGE),
    ([(0, 10, 0, 10, 0)], dict(hq=7), dsv.ERR_RANGE),
    ([(0, 10, 0, 10, 0)], dict(hq=1, hkv=2), dsv.ERR_RANGE),
    ([(0, 10, 0, 10, 0)], dict(hq=2048, hkv=8), dsv.ERR_RANGE),
    ([(0, 10, 0, 10, 0)], dict(d=96), dsv.ERR_RANGE),
    ([(95, 10, 0, 10, 0)], {}, dsv.ERR_LAYOUT),
    ([(0, 10, 95, 10, 0)], {}, dsv.ERR_LAYOUT),
    ([(-1, 10, 0, 10, 0)], {}, dsv.ERR_LAYOUT),
    ([(0, -1, 0, 10, 0)], {}, dsv.ERR_LAYOUT),
    ([(0, 10, -3, 10, 0)], {}, dsv.ERR_LAYOUT),
    ([(0, 10, 0, -10, 0)], {}, dsv.ERR_LAYOUT),
    ([(2 ** 31 - 5, 10, 0, 10, 0)], dict(nq=2 ** 31 - 1), dsv.ERR_LAYOUT),
    ([(20, 10, 0, 10, 0), (0, 21, 0, 10, 0)], {}, dsv.ERR_LAYOUT),
    ([(20, 10, 0, 10, 0), (25, 0, 0, 10, 0), (0, 20, 0, 10, 0)], {}, dsv.OK),
    ([(0, 10, 0, 10, 0)], dict(nq=-1), dsv.ERR_ARG),
    ([(0, 10, 0, 10, 0)], dict(nk=-1), dsv.ERR_ARG),
    ([(0, 2 ** 31 - 1, 0, 10, 0)], dict(nq=2 ** 31 - 1, hq=1024, hkv=1), dsv.ERR_SIZE),
])
def test_build(seqs, kw, want):
    assert build(seqs, **kw) == want


def test_build_refuses_null():
    n, h = ctypes.c_size_t(0), ctypes.c_void_p()
    assert lib.dsv_attn_build(None, 1, 10, 10, 2, 2, 64, ctypes.byref(n), ctypes.byref(h)) == dsv.ERR_ARG
    assert lib.dsv_attn_build(None, 0, 10, 10, 2, 2, 64, None, ctypes.byref(h)) == dsv.ERR_ARG
    assert lib.dsv_attn_build(None, 0, 10, 10, 2, 2, 64, ctypes.byref(n), None) == dsv.ERR_ARG
    assert lib.dsv_attn_train_rows(None, (ctypes.c_int64 * 2)()) == dsv.ERR_ARG
    assert lib.dsv_attn_workspace(None, 0, ctypes.byref(n)) == dsv.ERR_ARG
    lib.dsv_attn_free(None)


def test_train_rows_and_sizes():
    p = attn.Plan([(50, 20, 0, 30, 1), (0, 10, 0, 10, 0), (10, 5, 60, 7, 1)], 100, 100, 8, 2, 128)
    assert (p.train_q, p.train_k) == (25, 37)
    n = ctypes.c_size_t(0)
    assert lib.dsv_attn_workspace(p.handle, 7, ctypes.byref(n)) == dsv.ERR_RANGE
    assert attn.workspace_bytes(p, attn.torch.float32) >= 25 * 8 * 4
    with pytest.raises(dsv.DsvError):
        attn.Plan([(0, 10, 0, 10, 0)], 100, 100, 8, 3, 128)


BUF = 1 << 30  # an address that nothing reads: every call below is refused before a launch


def uploaded():
    """A plan that passes for one on the device."""
    p = attn.Plan([(0, 10, 0, 10, 1), (10, 1, 10, 2000, 0)], 11, 2010, 8, 2, 128)
    assert lib.dsv_attn_upload(p.handle, None, p.meta_bytes, None) == dsv.ERR_ARG
    assert lib.dsv_attn_upload(p.handle, BUF + 16, p.meta_bytes, None) == dsv.ERR_ARG
    assert lib.dsv_attn_upload(p.handle, BUF, p.meta_bytes - 1, None) == dsv.ERR_SIZE
    return p


def test_calls_refuse_a_plan_on_the_host():
    p = uploaded()
    v = [attn.View(BUF, 0, 0) for _ in range(8)]
    assert lib.dsv_attn_fwd(p.handle, 0, 0.1, *v[:4], BUF, BUF, 1 << 30, None) == dsv.ERR_ARG
    assert lib.dsv_attn_bwd(p.handle, 0, 0.1, *v[:4], BUF, *v[4:], BUF, 1 << 30, None) == dsv.ERR_ARG


def test_binding_refuses_wrong_tensors():
    torch = attn.torch
    p = attn.Plan([(0, 10, 0, 10, 1)], 10, 10, 4, 2, 64)
    q, k = torch.zeros((10, 4, 64)), torch.zeros((10, 2, 64))
    ws = torch.zeros(4096, dtype=torch.uint8)
    for bad in (dict(Q=q[:9]), dict(K=k.bfloat16()), dict(V=k.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(K=q), dict(lse=torch.zeros((10, 4)))):
        args = dict(dict(Q=q, K=k, V=k, O=q.clone()), **bad)
        with pytest.raises((TypeError, ValueError)):
            attn.fwd(p, args["Q"], args["K"], args["V"], O=args["O"], lse=args.get("lse"), workspace=ws)
    with pytest.raises(TypeError):
        attn.fwd(p, q.half(), k.half(), k.half(), O=q.half(), workspace=ws)
