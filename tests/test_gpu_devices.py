"""Tensors of a call in host memory beside others on the GPU are refused before the library sees an address."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_attention():
    from paper_2607_28848_amd import attn
    plan = attn.Plan([(0, 20, 0, 20, 1)], 20, 20, 4, 2, 64, device="cuda", window=5)
    q, k = torch.zeros((20, 4, 64), device="cuda"), torch.zeros((20, 2, 64), device="cuda")
    for bad in ((q.cpu(), k, k), (q, k.cpu(), k), (q, k, k.cpu()), (q.cpu(), k.cpu(), k.cpu())):
        with pytest.raises(ValueError):
            attn.fwd(plan, *bad)
    O, lse = attn.fwd(plan, q, k, k)
    with pytest.raises(ValueError):
        attn.fwd(plan, q, k, k, workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    for bad in (dict(O=O.cpu()), dict(lse=lse.cpu()), dict(dO=q.cpu()), dict(dQ=q.cpu())):
        with pytest.raises(ValueError):
            attn.bwd(plan, q, k, k, bad.get("O", O), bad.get("lse", lse), bad.get("dO", q), dQ=bad.get("dQ"))


def test_rotation():
    from paper_2607_28848_amd import rope
    q, pos, freq, w = torch.zeros((5, 4, 64), device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda"), \
        rope.frequencies(64, device="cuda"), torch.ones(64, device="cuda")
    for bad in (dict(pos=pos.cpu()), dict(freq=freq.cpu()), dict(q_weight=w.cpu()), dict(Q_out=q.cpu()), dict(Q=q.cpu())):
        args = dict(dict(Q=q, K=None, pos=pos, freq=freq, q_weight=w), **bad)
        with pytest.raises(ValueError):
            rope.fwd(**args)
    for bad in (dict(rows=pos.cpu()), dict(Q=q.cpu()), dict(dQ_out=q.cpu()), dict(dq_weight=w.cpu())):
        with pytest.raises(ValueError):
            rope.bwd(**dict(dict(dQ=q, dK=None, pos=pos, freq=freq, Q=q, q_weight=w), **bad))


def test_distillation():
    from paper_2607_28848_amd import vocab
    X, W, ids, t = torch.zeros((6, 64), device="cuda"), torch.zeros((50, 64), device="cuda"), \
        torch.zeros((6, 3), dtype=torch.int32, device="cuda"), torch.zeros((6, 3), device="cuda")
    for bad in (dict(X=X.cpu()), dict(W=W.cpu()), dict(ids=ids.cpu()), dict(teacher=t.cpu()), dict(weight=torch.ones(6)),
                dict(loss=torch.zeros(6)), dict(dX=X.cpu())):
        with pytest.raises(ValueError):
            vocab.distill_grad(**dict(dict(X=X, W=W, ids=ids, teacher=t), **bad))
