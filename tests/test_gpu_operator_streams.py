"""Attention and vocabulary-loss calls on a stream of their own while the current one is busy: what a call allocates
itself is filled and used on the call's stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def busy():
    """About 50 ms of work on the current stream."""
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    for _ in range(60):
        a = (a @ a) * 1e-2
    return a


def test_calls_on_their_own_stream():
    from paper_2607_28848_amd import attn, vocab
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((300, h, 64), generator=g).bfloat16().cuda() for h in (4, 2, 2))
    seqs = [(0, 200, 0, 200, 1), (200, 90, 200, 100, 0)]  # rows from 290 on belong to no sequence
    x, w = (torch.randn((n, 256), generator=g).bfloat16().cuda() for n in (70, 3000))
    target = torch.randint(3000, (70,), generator=g, dtype=torch.int32).cuda()

    def all_calls(stream=None):
        plan = attn.Plan(seqs, 300, 300, 4, 2, 64, device="cuda", stream=stream)
        o, lse = attn.fwd(plan, q, k, v, stream=stream)
        grads = attn.bwd(plan, q, k, v, o, lse, o[:200], stream=stream)
        return (o, lse, *grads, vocab.loss(x, w, target, stream=stream), *vocab.loss_grad(x, w, target, stream=stream))

    want = all_calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    keep = busy()
    got = all_calls(side)
    side.synchronize()
    first = [t.cpu() for t in got]
    torch.cuda.synchronize()
    assert all(torch.equal(a.cpu(), b) for a, b in zip(want, first))
    assert all(torch.equal(a, b) for a, b in zip(want, got))  # nothing came after them
    del keep
