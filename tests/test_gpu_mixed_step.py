"""The example's step -- linear layers, attention and vocabulary loss in one batch -- against autograd in 64 bits."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
REQUESTS = [(0, 37, 1, 0), (150, 20, 2, 0), (77, 1, 0, 0), (0, 70, 0, 1), (300, 1, 2, 0), (0, 33, 2, 1), (0, 1, 1, 1)]
RANKS = [16, 8, 32]


def load():
    spec = importlib.util.spec_from_file_location("mixed_step", os.path.join(ROOT, "examples", "mixed_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def block(dtype):
    n = sum(r[1] for r in REQUESTS)
    tokens = torch.randint(0, 500, (n,), generator=torch.Generator().manual_seed(3))
    return load().MixedStep(REQUESTS, RANKS, tokens, heads_q=4, heads_kv=2, head_dim=64, vocabulary=500, dtype=dtype)


def plain(b):
    """(hidden, scores, loss, {projection: (dA, dB)}) of the same step, from the formulas, in 64 bits on the CPU."""
    f = lambda t: t.detach().cpu().double()
    A = {n: f(t).requires_grad_() for n, t in b.A.items()}
    B = {n: f(t).requires_grad_() for n, t in b.B.items()}
    X = f(b.embedding)[b.tokens.cpu()]

    def lin(x, n):
        rows = []
        for s, l, a, _ in b.segments:
            r, xs = b.ranks[a], x[s:s + l]
            rows.append(xs @ f(b.W[n]).t() + (xs @ A[n][a, :r].t()) @ B[n][a, :, :r].t())
        return torch.cat(rows)

    q, k, v = (lin(X, n).unflatten(1, (-1, b.head_dim)) for n in "qkv")
    out = []
    for (s, l, k0, kl, _) in b.seqs:
        old = f(b.cache[:, k0:k0 + kl - l])
        ks, vs = (torch.cat([o, t[s:s + l]]).repeat_interleave(b.heads_q // b.heads_kv, dim=1) for o, t in zip(old, (k, v)))
        see = torch.arange(kl)[None, :] <= torch.arange(l)[:, None] + (kl - l)
        z = torch.einsum("qhd,khd->hqk", q[s:s + l], ks) / b.head_dim ** 0.5
        out.append(torch.einsum("hqk,khd->qhd", torch.where(see, z, -torch.inf).softmax(-1), vs).flatten(1))
    hidden = X + lin(torch.cat(out), "o")
    target = b.target.cpu().long()
    nll = -(hidden @ f(b.head).t()).log_softmax(-1).gather(1, target.clamp(min=0)[:, None])[:, 0]
    train = b.train.cpu()
    has = train[target[train] >= 0]
    loss = nll[has].mean()
    loss.backward()
    scores = nll[b.scored.cpu()].detach()
    return hidden.detach(), scores, float(loss.detach()), {n: (A[n].grad, B[n].grad) for n in A}


# Errors are relative to the tensor's largest value.  fp32: sums of at most 500 terms in each of the chain's nine products
# (u = 2^-24), so 9 * 500 u = 2.7e-4.  bf16: u = 2^-8 at each of the at most nine roundings of a path (q/k/v, p, O, Z,
# the sum, exponentials, dZ, dO, dq/dk/dv), each carried on by at most twice its size: 18 u = 7e-2.
TOL = {torch.float32: 2.7e-4, torch.bfloat16: 7e-2}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step_against_autograd(dtype):
    b = block(dtype)
    hidden, saved = b.forward()
    scores = b.score(hidden)
    loss, grads = b.backward(hidden, saved)
    want_hidden, want_scores, want_loss, want_grads = plain(b)

    def check(got, want, name):
        got = got.detach().cpu().double()
        err = float((got - want).abs().max() / want.abs().max())
        assert err <= TOL[dtype], "%s: %g" % (name, err)

    check(hidden, want_hidden, "hidden")
    check(scores, want_scores, "scores")
    assert abs(float(loss) - want_loss) <= TOL[dtype] * want_loss
    for n, (dA, dB) in want_grads.items():
        for a, r in enumerate(RANKS):
            check(grads[n][0][a, :r], dA[a, :r], "dA %s %d" % (n, a)) if dA[a, :r].any() else None
            check(grads[n][1][a, :, :r], dB[a, :, :r], "dB %s %d" % (n, a)) if dB[a, :, :r].any() else None


@pytest.mark.gpu
def test_loss_falls():
    b = block(torch.bfloat16)
    losses = []
    for _ in range(8):
        hidden, saved = b.forward()
        loss, grads = b.backward(hidden, saved)
        b.update(grads)
        losses.append(float(loss))
    assert losses[-1] < losses[0], losses
