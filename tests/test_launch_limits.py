"""Calls whose launches would have more work items than 32 bits count are refused for their size (CPU only: the addresses are
none, and a refused call reads nothing)."""
import ctypes

import pytest

from paper_2607_28848_amd import dsv, rope, vocab  # noqa: F401  (the bindings set the entries' argument types)
from paper_2607_28848_amd.attn import View

BUF = 1 << 40  # an address that nothing reads


@pytest.mark.parametrize("n,heads,d", [(1 << 26, 1, 64), ((1 << 26) + 5, 8, 128), ((1 << 31) - 1, 2, 64), (1 << 25, 64, 64)])
def test_rotation(n, heads, d):
    r = rope.Rope(n, heads, 0, d, 0, 0, 1e-6, None, None, None, None)
    v = View(BUF, 0, 0)
    out = View(BUF << 1, 0, 0)
    assert rope._lib.dsv_rope_fwd(1, ctypes.byref(r), ctypes.byref(v), None, None, None, 0, ctypes.byref(out), None, None,
                                  None) == dsv.ERR_SIZE


@pytest.mark.parametrize("T,k", [(1 << 18, 1024), (1 << 24, 1), ((1 << 23) + 1, 17), ((1 << 31) - 1, 1)])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("dtype", [0, 1])
def test_distillation(T, k, grad, dtype):
    lib, room = dsv.lib_handle(), (1 << 63) - 1
    if grad:
        rc = lib.dsv_vocab_distill_grad(dtype, T, 8, 40, k, BUF, 0, BUF, 0, None, 0, BUF, BUF, 1.0, None, None, BUF, 0, BUF, room, None)
    else:
        rc = lib.dsv_vocab_distill(dtype, T, 8, 40, k, BUF, 0, BUF, 0, BUF, BUF, 1.0, BUF, BUF, room, None)
    assert rc == dsv.ERR_SIZE


@pytest.mark.parametrize("T,V", [(1 << 24, 40), ((1 << 24) - 1, 1 << 24)])
def test_vocabulary_loss(T, V):
    lib, room = dsv.lib_handle(), (1 << 63) - 1
    assert lib.dsv_vocab_loss(0, T, 8, V, BUF, 0, BUF, 0, BUF, BUF, BUF, room, None) == dsv.ERR_SIZE
    assert lib.dsv_vocab_loss(1, T, 8, V, BUF, 0, BUF, 0, BUF, BUF, BUF, room, None) == dsv.ERR_SIZE
