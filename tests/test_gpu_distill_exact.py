"""What the distillation's other tests leave open: entries' logits that fp32 sums do not hold, references that move between the
pieces of the vocabulary, and the gradient against differences with a tolerance that an error of a few percent exceeds."""
import math

import pytest
import torch

from test_gpu_distill import check, make, oracle, run

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E32 = 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,K,V", [(3, 1024, 40), (150, 512, 200), (40, 4096, 64), (600, 256, 300)])
def test_entries_logits_are_summed_in_64_bits(dtype, T, K, V):
    """Every token is an entry and the teacher nearly the student.  The first eight columns put 2^17 and more into a logit and
    the last eight take it out again; in between are multiples of 2^-9, which a sum in fp32 loses beside that: such a logit
    is off by 2^-10 and more, a probability by a thousandth, as much as student and teacher differ.  Sums of eight products
    are exact (multiples of 2^-9 below 2^3, or of 2^7 below 2^19), so the entries' logits are, and with them loss and gradient: a
    probability is off by the exponent's rounding to fp32, its exponential and quotient, (|x - ref| ln 2 + 6) e with x within 64 of
    the reference, a share by e, and a sum of V products by V + 8 steps."""
    from paper_2607_28848_amd import vocab
    g = torch.Generator().manual_seed(K + V)

    def whole(n, *shape):
        return torch.randint(-n, n + 1, shape, generator=g).double()
    X, W = whole(7, T, K) / 64, whole(3, V, K) / 8
    X[:, :8] = 64 * (2048 + 16 * whole(31, T, 8))
    W[:, :8] = (1 + whole(1, V, 8).abs()) / 8
    X[:, -8:], W[:, -8:] = -X[:, :8], W[:, :8]
    assert torch.equal(X.to(dtype).double(), X) and torch.equal(W.to(dtype).double(), W)
    z = X @ W.t()
    short = torch.zeros((T, V))
    for c in range(K):
        short += X[:, c, None].float() * W[:, c].float()
    assert float((short.double() - z).abs().max()) > 2.0 ** -10
    ids = torch.rand((T, V), generator=g).argsort(1)
    teacher = (z.gather(1, ids) + 1e-3 * torch.randn((T, V), generator=g)).float()
    loss, dx = vocab.distill_grad(X.to(dtype).cuda(), W.to(dtype).cuda(), ids.int().cuda(), teacher.cuda())
    torch.cuda.synchronize()
    q, lq, lp = torch.softmax(teacher.double(), 1), torch.log_softmax(teacher.double(), 1), torch.log_softmax(z, 1).gather(1, ids)
    want = (q * (lq - lp)).sum(1)
    assert float((loss.cpu().double() - want).abs().max()) <= 2 * E32 * float(want.max()) + 2.0 ** -46 * float(z.abs().max())
    p, full = torch.softmax(z, 1), torch.zeros((T, V), dtype=torch.float64).scatter_(1, ids, q)
    value = (p - full) @ W
    bound = ((64 * 0.7 + 8) * E32 * ((p + full) @ W.abs()) + (V + 8) * E32 * ((p - full).abs() @ W.abs())
             + (2.0 ** -8 if dtype == BF else E32) * value.abs())
    check(dx, (value, 1.01 * bound + 1e-30), "dX")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_references_that_move_between_pieces(dtype):
    """Some rows' largest logits lie in a later piece, 100 and more (base 2) above everything before it: what was summed so far,
    the entries' part in it, is brought to the new reference.  Their entries lie before, at and behind the move."""
    from paper_2607_28848_amd import vocab
    T, K, V, k = (900, 64, 400000, 6) if dtype == BF else (900, 64, 200000, 6)
    g = torch.Generator(device="cuda").manual_seed(16)
    W = torch.randn((V, K), generator=g, device="cuda") * 0.25
    X = torch.randn((T, K), generator=g, device="cuda")
    width = (256 << 20) // (2 if dtype == BF else 4) // T
    late = [width + width // 2, V - 3, width + 5, V - width // 3]
    assert width < V / 2 and min(late) > width
    for row, at in enumerate(late):
        W[at] = X[row] * (90.0 / float((X[row] ** 2).sum()))  # a logit of 90
    W, X = W.to(dtype), X.to(dtype)
    ids = torch.randint(V, (T, k), generator=g, device="cuda", dtype=torch.int32)
    for row, at in enumerate(late):
        ids[row] = torch.tensor([3, at, width - 1, at + 1, V - 1, width // 256 * 256], dtype=torch.int32)
    ids[1, 1] = 77  # the largest token is no entry
    teacher = torch.randn((T, k), generator=g, device="cuda")
    for row in (0, 2, 3):
        teacher[row, 1] += 60.0
    loss, dx = vocab.distill_grad(X, W, ids, teacher)
    alone = vocab.distill(X, W, ids, teacher)
    torch.cuda.synchronize()
    rows = torch.cat((torch.arange(6), torch.arange(T - 2, T))).cuda()
    z = X[:4].double() @ W.double().t()
    assert all(float(z[i].max() - z[i, :width // 2].max()) > 60 * math.log(2) for i in range(4))
    loss_w, dx_w = oracle(X[rows], W, ids[rows], teacher[rows], 1.0, None)
    check(loss[rows], loss_w, "loss")
    check(alone[rows], loss_w, "loss alone")
    check(dx[rows], dx_w, "dX")


@pytest.mark.parametrize("along", [True, False])
def test_gradient_against_differences(along):
    """fp32, central differences of the weighted losses' sum, along the gradient and along a random direction.  The tolerance:
    what the same differences are off in 64 bits, the losses' bounds over 2 h, and the gradient's own; a few percent of the
    derivative along the gradient."""
    from paper_2607_28848_amd import vocab
    X, W, ids, teacher, weight = make(30, 64, 400, 7, F32, seed=9)
    tau, h = 1.5, 2.0 ** -5
    _, dx = vocab.distill_grad(X, W, ids, teacher, temperature=tau, weight=weight)
    u = dx * (math.sqrt(dx.numel()) / float(dx.norm())) if along else torch.randn(X.shape, generator=torch.Generator().manual_seed(2)).cuda()
    up, down = X + h * u, X - h * u
    step = (up.double() - down.double()) / (2 * h)  # the direction as rounded
    losses = [vocab.distill(x, W, ids, teacher, temperature=tau).double() for x in (up, down)]
    num = float(((losses[0] - losses[1]) * weight.double()).sum()) / (2 * h)
    torch.cuda.synchronize()
    (lu, bu), _ = oracle(up, W, ids, teacher, tau, weight)
    (ld, bd), _ = oracle(down, W, ids, teacher, tau, weight)
    _, (value, bound) = oracle(X, W, ids, teacher, tau, weight)
    w, s = weight.cpu().double(), step.cpu()
    exact = float((value * s).sum())
    tolerance = abs(float(((lu - ld) * w).sum()) / (2 * h) - exact) + float((w.abs() * (bu + bd)).sum()) / (2 * h) + float((bound * s.abs()).sum())
    ana = float((dx.cpu().double() * s).sum())
    print(num, ana, exact, tolerance, flush=True)
    if along:
        assert tolerance < 0.05 * abs(exact)
    assert abs(num - ana) <= tolerance


@pytest.mark.parametrize("T,V,k", [(300, 131080, 1024), (130, 131072, 999), (257, 131072, 3), (100, 131080, 1023), (17, 131072, 1)])
def test_entries_of_whole_tiles(T, V, k):
    """bf16 tiles of 256 and 128 rows and 256 columns with many entries and few, at the tiles' first and last columns among them."""
    X, W, ids, teacher, weight = make(T, 64, V, k, BF, seed=21)
    edges = torch.tensor([0, 255, 256, V - 1, 511, 512, 65535, 65536], dtype=torch.int32)[:k].cuda()
    ids[::3, :len(edges)] = edges
    ids[T - 1, 0] = V - 1
    run(X, W, ids, teacher, 1.0, weight)
