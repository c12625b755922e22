"""Logits of -infinity in the vocabulary loss: they drop out of the losses, and of the gradients but for the head's
infinite elements themselves, where 0 times them is NaN as it is in softmax(z) W."""
import math

import pytest
import torch

from test_gpu_vocab import BF, F32, check, make, oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,K,V", [(5, 64, 300), (70, 72, 1032), (300, 136, 5000), (130, 64, 33008)])
def test_logits_of_minus_infinity(dtype, T, K, V):
    """A tenth of the head's rows, whole tiles of columns and the first and the last column among them; the targets lie
    elsewhere."""
    from paper_2607_28848_amd import vocab
    X, W, target, weight = make(T, K, V, dtype, seed=V)
    X[:, 0] = 0.5 + X[:, 0].abs()
    gone = torch.rand(V, generator=torch.Generator().manual_seed(1)) < 0.1
    gone[0] = gone[V - 1] = True
    gone[V // 2:V // 2 + V // 8] = True
    gone, kept = gone.nonzero()[:, 0].cuda(), (~gone).nonzero()[:, 0].cuda()
    target = kept[target.long() % kept.numel()].to(torch.int32)
    W[gone, 0] = -math.inf
    place = torch.full((V,), -1, dtype=torch.int32, device="cuda")
    place[kept] = torch.arange(kept.numel(), dtype=torch.int32, device="cuda")
    want_loss, (dx, bound) = oracle(X, W[kept], place[target.long()], weight)
    check(vocab.loss(X, W, target), want_loss, "loss alone")
    for Wt in (None, W.t().contiguous()):
        loss, got = vocab.loss_grad(X, W, target, weight=weight, Wt=Wt)
        check(loss, want_loss, "loss")
        check(got[:, 1:], (dx[:, 1:], bound[:, 1:]), "dX")
        assert bool(got[:, 0].isnan().all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_targets_of_minus_infinity(dtype):
    """A target that cannot be: an infinite loss, for its row alone."""
    from paper_2607_28848_amd import vocab
    X, W, target, _ = make(40, 64, 500, dtype, seed=2)
    X[:, 0] = 0.5 + X[:, 0].abs()
    W[7, 0] = -math.inf
    target[target == 7] = 8
    target[[3, 33]] = 7
    loss = vocab.loss(X, W, target)
    assert bool((loss.isinf() == (target == 7)).all()) and bool((loss[[3, 33]] > 0).all())
