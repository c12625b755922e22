"""The example's step -- linear layers, norms and rotation into a cache, windowed attention, distillation, and back -- against
autograd in 64 bits, and captured into a graph."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
REQUESTS = [(0, 37, 1, 0), (150, 20, 2, 0), (77, 1, 0, 0), (0, 70, 0, 1), (300, 1, 2, 0), (0, 33, 2, 1), (0, 1, 1, 1)]
RANKS = [16, 8, 32]
pytestmark = pytest.mark.gpu


def block(dtype):
    spec = importlib.util.spec_from_file_location("distill_step", os.path.join(ROOT, "examples", "distill_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    n = sum(r[1] for r in REQUESTS)
    tokens = torch.randint(0, 500, (n,), generator=torch.Generator().manual_seed(3))
    return m.DistillStep(REQUESTS, RANKS, tokens, window=23, sinks=3, heads_q=4, heads_kv=2, head_dim=64, vocabulary=500, dtype=dtype)


def plain(b):
    """(hidden, loss, {projection: (dA, dB)}, norm gradients) of the same step, from the formulas, in 64 bits on the CPU."""
    f = lambda t: t.detach().cpu().double()
    A = {n: f(t).requires_grad_() for n, t in b.A.items()}
    B = {n: f(t).requires_grad_() for n, t in b.B.items()}
    norms = [f(t).requires_grad_() for t in (b.q_norm, b.k_norm)]
    X = f(b.embedding)[b.tokens.cpu()]

    def lin(x, n):
        rows = []
        for s, l, a, _ in b.segments:
            r, xs = b.ranks[a], x[s:s + l]
            rows.append(xs @ f(b.W[n]).t() + (xs @ A[n][a, :r].t()) @ B[n][a, :, :r].t())
        return torch.cat(rows)

    def rotated(x, w):
        x = x * w / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        t = (f(b.pos)[:, None] * f(b.freq)[None, :])[:, None, :]
        u, v = x.chunk(2, -1)
        return torch.cat((u * t.cos() - v * t.sin(), v * t.cos() + u * t.sin()), -1)

    q, k, v = (lin(X, n).unflatten(1, (-1, b.head_dim)) for n in "qkv")
    q, k = rotated(q, norms[0]), rotated(k, norms[1])
    out = []
    for (s, l, k0, kl, _) in b.seqs:
        old = f(b.cache[:, k0:k0 + kl - l])
        ks, vs = (torch.cat([o, t[s:s + l]]).repeat_interleave(b.heads_q // b.heads_kv, dim=1) for o, t in zip(old, (k, v)))
        j, p = torch.arange(kl)[None, :], torch.arange(l)[:, None] + (kl - l)
        see = (j <= p) & ((j > p - b.window) | (j < b.sinks))
        z = torch.einsum("qhd,khd->hqk", q[s:s + l], ks) / b.head_dim ** 0.5
        out.append(torch.einsum("hqk,khd->qhd", torch.where(see, z, -torch.inf).softmax(-1), vs).flatten(1))
    hidden = X + lin(torch.cat(out), "o")
    tau = b.temperature
    logp = (hidden[b.train.cpu()] @ f(b.head).t() / tau).log_softmax(-1)
    ids = b.ids.cpu().long()
    has = ids[:, 0] >= 0
    logq = (f(b.teacher) / tau).log_softmax(-1)
    loss = tau ** 2 * (logq.exp() * (logq - logp.gather(1, ids.clamp(min=0)))).sum(1)[has].mean()
    loss.backward()
    return hidden.detach(), float(loss.detach()), {n: (A[n].grad, B[n].grad) for n in A}, [t.grad for t in norms]


# Errors are relative to the tensor's largest value, as in the plain step's test.  fp32: sums of at most 500 terms in each of
# eleven products and norms (u = 2^-24): 11 * 500 u = 3.3e-4.  bf16: u = 2^-8 at each of the at most twelve roundings of a
# path (q/k/v, their rotation, p, O, Z, the sum, exponentials, dZ, dO, dq/dk/dv, their rotation back and the products' operands),
# each carried on by at most twice its size: 24 u = 9.4e-2.
TOL = {torch.float32: 3.3e-4, torch.bfloat16: 9.4e-2}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step_against_autograd(dtype):
    b = block(dtype)
    hidden, saved = b.forward()
    loss, grads, norms = b.backward(hidden, saved)
    want_hidden, want_loss, want_grads, want_norms = plain(b)

    def check(got, want, name):
        got = got.detach().cpu().double()
        err = float((got - want).abs().max() / want.abs().max())
        assert err <= TOL[dtype], "%s: %g" % (name, err)

    check(hidden, want_hidden, "hidden")
    assert abs(float(loss) - want_loss) <= TOL[dtype] * want_loss
    check(norms[0], want_norms[0], "q norm")
    check(norms[1], want_norms[1], "k norm")
    for n, (dA, dB) in want_grads.items():
        for a, r in enumerate(RANKS):
            check(grads[n][0][a, :r], dA[a, :r], "dA %s %d" % (n, a)) if dA[a, :r].any() else None
            check(grads[n][1][a, :, :r], dB[a, :, :r], "dB %s %d" % (n, a)) if dB[a, :, :r].any() else None


def test_steps_run():
    b = block(torch.bfloat16)
    for _ in range(3):
        hidden, saved = b.forward()
        loss, grads, _ = b.backward(hidden, saved)
        b.update(grads)
        assert bool(torch.isfinite(loss)) and all(bool(torch.isfinite(g).all()) for p in grads.values() for g in p)


def test_step_in_a_graph():
    """The forward and backward of the new operators captured once and replayed, with other eager steps in between: the
    same bits as the eager step's."""
    b = block(torch.bfloat16)
    hidden, saved = b.forward()
    b.backward(hidden, saved)  # the library's side streams and the allocator's blocks exist before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hidden, saved = b.forward()
        loss, grads, norms = b.backward(hidden, saved)
    for i in range(3):
        b.q_norm.mul_(1.01)
        b.teacher.add_(0.1 * i * b.teacher.roll(1, 1))
        graph.replay()
        torch.cuda.synchronize()
        eager_hidden, eager_saved = b.forward()
        eager_loss, eager_grads, eager_norms = b.backward(eager_hidden, eager_saved)
        torch.cuda.synchronize()
        assert torch.equal(hidden, eager_hidden) and torch.equal(loss, eager_loss)
        for n in eager_grads:
            for a, r in enumerate(RANKS):  # what lies behind a rank, and adapters without samples, are not written
                if a in [s[2] for s in b.segments if s[3]]:
                    assert torch.equal(grads[n][0][a, :r], eager_grads[n][0][a, :r])
                    assert torch.equal(grads[n][1][a, :, :r], eager_grads[n][1][a, :, :r])
        assert all(torch.equal(x, y) for x, y in zip(norms, eager_norms))
