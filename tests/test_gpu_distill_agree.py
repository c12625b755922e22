"""Losses of students that agree with their teacher, against the definition in 64 bits: near 0 they keep their accuracy, and
are never below it where a row's entries name different tokens.

Bounds, e = 2^-24.  An entry's own logit over the temperature is off by at most d = 8 e sum|x||w| / tau (eight products a sum
in fp32, the rest in 64 bits), another token's by m as in the other tests (the products' K-long fp32 sums, and the exponent's
factor): m = ((K + 4) sum|x||w| / tau + 4 |z|) e.  With p' the student's share of its entries' mass S and R the mass of the
others, the loss is KL(q || p') + log(1 + R / S).  Its first part moves by at most d sum|p' - q| + d^2, its second by R / S times the
relative error of R and S, 2 (m + d) + (V + 40) e for the exponentials' sum; 64-bit steps leave 2^-46 of the logits; the loss is
rounded once."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E32 = 2.0 ** -24


def make(T, K, V, k, dtype, tau, std, far, seed):
    """Rows whose entries are their largest logits, with the teacher's a little off the student's: `far` of them, 0 for a
    teacher that differs by its logits' rounding to fp32 alone."""
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn((V, K), generator=g) * std * tau / math.sqrt(K)).to(dtype)
    X = torch.randn((T, K), generator=g).to(dtype)
    z = X.double() @ W.double().t() / tau
    ids = z.topk(k, 1).indices
    ids = ids.gather(1, torch.rand((T, k), generator=g).argsort(1))
    teacher = z.gather(1, ids) * tau + 5.0 + far * torch.randn((T, k), generator=g)
    return X, W, ids, teacher.float(), z


def oracle(X, W, ids, teacher, tau, z):
    K, V = X.shape[1], W.shape[0]
    q, lq = (f(teacher.double() / tau, 1) for f in (torch.softmax, torch.log_softmax))
    own = z.gather(1, ids)
    lp = torch.log_softmax(own, 1)
    apart = z.scatter(1, ids, -math.inf)
    rest = torch.exp(torch.logsumexp(apart, 1) - torch.logsumexp(own, 1))  # R / S
    loss = torch.where(q > 0, q * (lq - lp), 0.0).sum(1) + torch.log1p(rest)
    size = X.abs().double() @ W.abs().double().t() / tau
    d = (8 * E32 * size).gather(1, ids).amax(1)
    m = (((K + 4) * size + 4 * z.abs()) * E32).amax(1)
    bound = d * (torch.exp(lp) - q).abs().sum(1) + d * d + rest * (2 * (m + d) + (V + 40) * E32)
    return loss, 1.01 * (bound + E32 * loss) + 2.0 ** -46 * z.abs().amax(1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", [0.0, 1e-3, 0.1])
@pytest.mark.parametrize("T,K,V,k,tau,std", [(1, 64, 700, 40, 1.0, 12.0), (70, 128, 3000, 64, 2.0, 10.0), (300, 64, 515, 200, 1.0, 9.0),
                                             (5, 512, 9000, 1024, 1.0, 8.0), (600, 72, 2049, 7, 1.0, 30.0), (40, 64, 64, 64, 0.5, 6.0)])
def test_losses_near_zero(dtype, far, T, K, V, k, tau, std):
    from paper_2607_28848_amd import vocab
    print(dtype, far, T, K, V, k, flush=True)
    X, W, ids, teacher, z = make(T, K, V, k, dtype, tau, std, far, seed=T + k)
    want, bound = oracle(X, W, ids, teacher, tau, z)
    if far < 0.1 and k > 7:
        assert float(want.median()) < 1e-4 and float((bound / want.clamp_min(1e-6)).median()) < 0.05
    args = (X.cuda(), W.cuda(), ids.int().cuda(), teacher.cuda())
    alone = vocab.distill(*args, temperature=tau)
    loss, _ = vocab.distill_grad(*args, temperature=tau)
    torch.cuda.synchronize()
    for got in (alone, loss):
        got = got.cpu().double()
        assert bool((got >= 0).all()), float(got.min())
        off = (got - want).abs()
        assert bool((off <= bound).all()), (float((off / bound).max()), float(off.max()))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_repeated_tokens_may_go_below(dtype):
    """Two entries of one token, each with half its share: sum q log q falls by log 2 and so does the loss."""
    from paper_2607_28848_amd import vocab
    X, W, ids, teacher, z = make(9, 64, 300, 300, dtype, 1.0, 4.0, 0.0, seed=1)
    want, bound = oracle(X, W, ids, teacher, 1.0, z)
    twice = torch.cat((ids, ids), 1).int().cuda(), torch.cat((teacher, teacher), 1).cuda()
    loss = vocab.distill(X.cuda(), W.cuda(), *twice)
    torch.cuda.synchronize()
    off = (loss.cpu().double() - (want - math.log(2))).abs()
    assert bool((off <= bound + 2 * E32).all()) and float(loss.max()) < 0
