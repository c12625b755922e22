"""Where the tensors of a call have to be (CPU only, the devices are stand-ins): on the device of the call's stream, which need
not be the current one; pinned host memory may stand beside a GPU's."""
import types

import pytest
import torch

from paper_2607_28848_amd import _marshal, attn


def stream(index, handle=1000):
    s = types.SimpleNamespace(cuda_stream=handle)
    if index is not None:
        s.device = torch.device("cuda", index)
    return s


@pytest.fixture
def at(monkeypatch):
    """here() of tensors that are on the GPU of that number, beside a current one of number 0."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def call(index, **how):
        monkeypatch.setattr(attn, "_marshal", types.SimpleNamespace(where=lambda *t: index))
        return attn.here(None, **how)
    return call


def test_a_stream_of_another_device_takes_that_device_s_tensors(at):
    assert at(1, stream=stream(1)) is False and at(0, stream=stream(0)) is False
    assert at(0) is False and at(3, stream=stream(None)) is False
    for index, how in ((1, {}), (0, dict(stream=stream(1))), (1, dict(stream=stream(0))),
                       (1, dict(stream=stream(1, handle=0))), (1, dict(stream=stream(None, handle=0)))):
        with pytest.raises(ValueError):
            at(index, **how)


def test_host_memory(at):
    assert at(-1) is True and at(-1, stream=stream(1)) is True and at(-2) is False


def test_where():
    assert _marshal.where(torch.zeros(3), None, torch.zeros(0)) == -1
    assert _marshal.where() == -2 and _marshal.where(None, torch.zeros(0)) == -2
    with pytest.raises(ValueError):
        _marshal.where(torch.zeros(3), torch.zeros(0, device="meta"))


@pytest.mark.gpu
def test_pinned_tensors_beside_the_gpus():
    """The log-sum-exp of an attention call kept in pinned memory, a loss's targets read from it."""
    from paper_2607_28848_amd import vocab
    gen = torch.Generator().manual_seed(1)
    plan = attn.Plan([(0, 20, 0, 20, 1)], 20, 20, 4, 2, 64, device="cuda")
    q, k = torch.randn((20, 4, 64), generator=gen).cuda(), torch.randn((20, 2, 64), generator=gen).cuda()
    O, lse = attn.fwd(plan, q, k, k)
    kept = torch.zeros((4, 20), pin_memory=True)
    P, _ = attn.fwd(plan, q, k, k, lse=kept)
    torch.cuda.synchronize()
    assert torch.equal(P, O) and torch.equal(kept, lse.cpu())
    a, b = attn.bwd(plan, q, k, k, O, lse, q), attn.bwd(plan, q, k, k, O, kept, q)
    X, W = torch.randn((6, 64), generator=gen).cuda(), torch.randn((50, 64), generator=gen).cuda()
    target = torch.tensor([3, 1, 49, -1, 0, 7], dtype=torch.int32, pin_memory=True)
    losses = vocab.loss(X, W, target), vocab.loss(X, W, target.cuda())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(*losses)
    assert _marshal.where(q, kept) == 0 and _marshal.where(kept) == -2


@pytest.mark.gpu
def test_the_loss_refuses_what_the_other_calls_refuse():
    from paper_2607_28848_amd import vocab
    X, W, target = torch.zeros((6, 64)), torch.zeros((50, 64)), torch.zeros(6, dtype=torch.int32)
    calls = [lambda x, w, t, **how: vocab.loss(x, w, t, **how), lambda x, w, t, **how: vocab.loss_grad(x, w, t, **how)]
    for call in calls:
        for bad in ((X, W.cuda(), target.cuda()), (X.cuda(), W, target.cuda()), (X.cuda(), W.cuda(), target), (X, W, target)):
            with pytest.raises(ValueError):
                call(*bad)
        with pytest.raises(ValueError):
            call(X.cuda(), W.cuda(), target.cuda(), loss=torch.zeros(6))
    with pytest.raises(ValueError):
        vocab.loss_grad(X.cuda(), W.cuda(), target.cuda(), dX=X.clone())
