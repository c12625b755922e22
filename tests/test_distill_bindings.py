"""What the distillation's calls refuse (CPU only): every call here is refused before a launch, or has no rows."""
import ctypes
import types

import pytest
import torch

from paper_2607_28848_amd import dsv, vocab

NONE = dict(workspace=torch.zeros(0, dtype=torch.uint8), stream=types.SimpleNamespace(cuda_stream=0))
BUF = 1 << 30  # an address that nothing reads


def call(grad=True, **changed):
    t = dict(X=torch.zeros((6, 16)), W=torch.zeros((8, 16)), ids=torch.zeros((6, 3), dtype=torch.int32), teacher=torch.zeros((6, 3)),
             loss=torch.zeros(6))
    if grad:
        t.update(dX=torch.zeros((6, 16)))
    t.update(changed)
    return (vocab.distill_grad if grad else vocab.distill)(**NONE, **t)


@pytest.mark.parametrize("grad", [True, False])
def test_the_calls_as_they_are_reach_the_library(grad):
    with pytest.raises(dsv.DsvError):
        call(grad)


@pytest.mark.parametrize("changed", [
    dict(ids=torch.zeros((6, 3), dtype=torch.int64)), dict(ids=torch.zeros((5, 3), dtype=torch.int32)), dict(teacher=torch.zeros((6, 4))),
    dict(teacher=torch.zeros((6, 3), dtype=torch.bfloat16)), dict(teacher=torch.zeros((3, 6)).t()),
    dict(ids=torch.zeros((6, 6), dtype=torch.int32)[:, ::2]), dict(X=torch.zeros((1, 16)).expand(6, 16)),
    dict(W=torch.zeros((1, 16)).expand(8, 16)), dict(loss=torch.zeros(5)), dict(ids=torch.zeros((6, 3), dtype=torch.int32, device="meta"))])
@pytest.mark.parametrize("grad", [True, False])
def test_binding_refuses(changed, grad):
    with pytest.raises(ValueError):
        call(grad, **changed)


@pytest.mark.parametrize("changed", [dict(dX=torch.zeros((1, 16)).expand(6, 16)), dict(Wt=torch.zeros((1, 8)).expand(16, 8)),
                                     dict(weight=torch.zeros(5)), dict(weight=torch.zeros(6, dtype=torch.float64))])
def test_binding_refuses_the_gradients(changed):
    with pytest.raises(ValueError):
        call(True, **changed)


def test_types():
    for changed in (dict(X=torch.zeros((6, 16), dtype=torch.float16)), dict(W=torch.zeros((8, 16), dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            call(True, **changed)


def test_workspace():
    lib, n = dsv.lib_handle(), ctypes.c_size_t(0)
    plain = vocab.workspace_bytes(100, 64, 5000, torch.float32, True)
    assert vocab.distill_workspace_bytes(100, 64, 5000, 7, torch.float32, True) >= plain + 100 * 7 * 12 + 800
    assert lib.dsv_vocab_distill_workspace(0, 5, 64, 100, 0, 0, 1, ctypes.byref(n)) == dsv.ERR_SIZE
    assert lib.dsv_vocab_distill_workspace(0, 5, 64, 100, 1025, 0, 1, ctypes.byref(n)) == dsv.ERR_SIZE
    assert lib.dsv_vocab_distill_workspace(0, 5, 64, 100, 3, 0, 1, None) == dsv.ERR_ARG
    assert lib.dsv_vocab_distill_workspace(2, 5, 64, 100, 3, 0, 1, ctypes.byref(n)) == dsv.ERR_RANGE
    assert lib.dsv_vocab_distill_workspace(0, -1, 64, 100, 3, 0, 1, ctypes.byref(n)) == dsv.ERR_ARG
    assert lib.dsv_vocab_distill_workspace(0, 5, 60, 100, 3, 0, 1, ctypes.byref(n)) == dsv.ERR_SIZE
    with pytest.raises(ValueError):
        vocab.distill_workspace_bytes(5, 64, 100, 1 << 32, torch.float32, True)
    # rows times entries past 32 bits
    assert vocab.distill_workspace_bytes(1 << 30, 8, 8, 1024, torch.float32, False) > 12 << 40


def test_c_entries():
    lib = dsv.lib_handle()

    def go(T=5, K=64, V=100, k=3, X=BUF, ldx=0, W=BUF, ldw=0, ids=BUF, teacher=BUF, tau=1.0, loss=BUF, ws=BUF, n=1 << 40, dt=0):
        return lib.dsv_vocab_distill(dt, T, K, V, k, X, ldx, W, ldw, ids, teacher, tau, loss, ws, n, None)

    def back(T=5, K=64, V=100, k=3, X=BUF, W=BUF, Wt=None, ldwt=0, ids=BUF, teacher=BUF, tau=1.0, weight=None, loss=None, dX=BUF, lddx=0,
             ws=BUF, n=1 << 40, dt=0):
        return lib.dsv_vocab_distill_grad(dt, T, K, V, k, X, 0, W, 0, Wt, ldwt, ids, teacher, tau, weight, loss, dX, lddx, ws, n, None)

    for f in (go, back):
        for kw, want in ((dict(T=-1), dsv.ERR_ARG), (dict(X=None), dsv.ERR_ARG), (dict(X=BUF + 8), dsv.ERR_ARG), (dict(W=None), dsv.ERR_ARG),
                         (dict(ids=None), dsv.ERR_ARG), (dict(ids=BUF + 2), dsv.ERR_ARG), (dict(teacher=None), dsv.ERR_ARG),
                         (dict(teacher=BUF + 1), dsv.ERR_ARG), (dict(ws=None), dsv.ERR_ARG), (dict(ws=BUF + 64), dsv.ERR_ARG),
                         (dict(n=100), dsv.ERR_SIZE), (dict(k=0), dsv.ERR_SIZE), (dict(k=1025), dsv.ERR_SIZE), (dict(K=12), dsv.ERR_SIZE),
                         (dict(V=0), dsv.ERR_SIZE), (dict(dt=5), dsv.ERR_RANGE), (dict(tau=0.0), dsv.ERR_RANGE), (dict(tau=-1.0), dsv.ERR_RANGE),
                         (dict(tau=float("nan")), dsv.ERR_RANGE), (dict(tau=float("inf")), dsv.ERR_RANGE), (dict(tau=1e-39), dsv.ERR_RANGE),
                         (dict(tau=1e39), dsv.ERR_RANGE), (dict(tau=1e-310), dsv.ERR_RANGE)):
            assert f(**kw) == want, kw
        assert f(T=0, X=None, ids=None, teacher=None, **(dict(loss=None) if f is go else dict(dX=None))) == dsv.OK
    assert go(loss=None) == dsv.ERR_ARG and go(ldx=60) == dsv.ERR_SIZE and go(ldw=68) == dsv.ERR_SIZE
    assert back(dX=None) == dsv.ERR_ARG and back(lddx=60) == dsv.ERR_SIZE and back(weight=BUF + 2) == dsv.ERR_ARG
    assert back(loss=BUF + 1) == dsv.ERR_ARG and back(Wt=BUF + 8, V=104) == dsv.ERR_ARG and back(Wt=BUF, ldwt=100, V=104) == dsv.ERR_SIZE
