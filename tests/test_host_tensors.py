"""Calls whose tensors are all in host memory, on a machine with a GPU, are refused before the library is called: its kernels
would read host addresses.  The machine and the library's entries are stand-ins: nothing is ever launched."""
import types

import pytest
import torch

from paper_2607_28848_amd import dsv, rope, vocab

STREAM = types.SimpleNamespace(cuda_stream=0)
POS = torch.zeros(6, dtype=torch.int32)
FREQ = torch.zeros(16, dtype=torch.float64)


@pytest.fixture
def entered(monkeypatch):
    """The library's entries that were called."""
    seen = []

    class Entries:
        def __getattr__(self, name):
            return lambda *a: seen.append(name) or 0
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(rope, "_fwd", Entries().rope_fwd)
    monkeypatch.setattr(rope, "_bwd", Entries().rope_bwd)
    monkeypatch.setattr(vocab, "_lib", Entries())
    return seen


def forward(n=6):
    x = torch.zeros((n, 2, 64))
    return rope.fwd(x, None, POS[:n], FREQ, Q_out=x.clone(), stream=STREAM)


def backward(m=6, **how):
    x = torch.zeros((m, 2, 64))
    return rope.bwd(x, None, POS, FREQ, rows=POS[:m], dQ_out=x.clone(),
                    workspace=torch.zeros(256, dtype=torch.uint8), stream=STREAM, **how)


def distill(grad, T=6):
    X, ids = torch.zeros((T, 16)), torch.zeros((T, 3), dtype=torch.int32)
    how = dict(loss=torch.zeros(T), workspace=torch.zeros(256, dtype=torch.uint8), stream=STREAM)
    if grad:
        return vocab.distill_grad(X, torch.zeros((8, 16)), ids, torch.zeros((T, 3)), dX=X.clone(), **how)
    return vocab.distill(X, torch.zeros((8, 16)), ids, torch.zeros((T, 3)), **how)


CALLS = [forward, backward, lambda: backward(0, Q=torch.zeros((6, 2, 64)), q_weight=torch.ones(64), dq_weight=torch.zeros(64)),
         lambda: distill(False), lambda: distill(True)]


@pytest.mark.parametrize("call", CALLS)
def test_refused(entered, call):
    for kind in (ValueError, dsv.DsvError):
        with pytest.raises(kind, match="host memory"):
            call()
    assert not entered


@pytest.mark.parametrize("call", [lambda: forward(0), lambda: backward(0), lambda: distill(False, 0), lambda: distill(True, 0)])
def test_without_rows_there_is_nothing_to_refuse(entered, call):
    call()
    assert len(entered) == 1


def test_other_refusals_come_first(entered):
    with pytest.raises(TypeError):
        rope.fwd(torch.zeros((6, 2, 64)), None, POS, FREQ, Q_out=torch.zeros((6, 2, 64), dtype=torch.float16), stream=STREAM)
    with pytest.raises(TypeError):
        vocab.distill(torch.zeros((6, 16)), torch.zeros((8, 16), dtype=torch.float16), torch.zeros((6, 3), dtype=torch.int32),
                      torch.zeros((6, 3)), loss=torch.zeros(6), stream=STREAM)
    assert not entered


@pytest.mark.parametrize("call", CALLS)
def test_without_a_gpu_the_library_answers(entered, call, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_available", lambda: False)
    call()
    assert len(entered) == 1


@pytest.mark.parametrize("grad", [False, True])
def test_the_loss_refuses_them_too(entered, grad):
    def call(T):
        X, how = torch.zeros((T, 16)), dict(loss=torch.zeros(T), workspace=torch.zeros(256, dtype=torch.uint8), stream=STREAM)
        if grad:
            how["dX"] = X.clone()
        (vocab.loss_grad if grad else vocab.loss)(X, torch.zeros((8, 16)), POS[:T], **how)
    with pytest.raises(ValueError, match="host memory"):
        call(6)
    assert not entered
    call(0)
    assert len(entered) == 1
