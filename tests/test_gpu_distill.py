"""Distillation on the GPU against the definition in 64 bits: entries from one to a thousand, padding, repeated and masked
entries, temperatures, several pieces, strides, streams and graphs, gradients, and its step beside the other operators.

Bounds are first-order worst cases, as in the vocabulary loss's tests: u is 2^-8 in bf16 and 2^-24 in fp32, e = 2^-24.  A
logit over the temperature is off by at most ez = ((K + 4) sum|x||w| + 4 |z|) e / tau, m is the row's largest ez, a
probability's relative error is at most r = 2 m + (V + 32) e + 4 e max|z| / tau, and that of a term as an operand u more; the
teacher's tokens are no operands.  Their shares are rounded once, and the entries' sum takes k + 8 steps."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E32 = 2.0 ** -24


def oracle(X, W, ids, teacher, tau, weight):
    u = 2.0 ** -8 if X.dtype == BF else E32
    x, w, t = X.detach().cpu().double(), W.detach().cpu().double(), teacher.detach().cpu().double() / tau
    ids = ids.cpu().long()
    T, K = x.shape
    V, k = w.shape[0], ids.shape[1]
    keep = (ids >= 0) & (ids < V)
    t = torch.where(keep, t, -math.inf)
    has = t.amax(1) > -math.inf
    x = torch.where(has[:, None], x, 0.0)
    at = torch.where(keep, ids, 0)
    q = torch.where(has[:, None], torch.softmax(torch.where(has[:, None], t, 0.0), 1), 0.0)
    z = x @ w.t() / tau
    m = (((K + 4) * (x.abs() @ w.abs().t()) / tau + 4 * z.abs()) * E32).amax(1)
    logp = torch.log_softmax(z, 1)
    p = torch.exp(logp)
    loss = torch.where(q > 0, q * (torch.log(q) - logp.gather(1, at)), 0.0).sum(1)
    lb = 1.05 * (2 * m + (V + 40) * E32 + 4 * E32 * loss.abs()) * has + 1e-30
    r = 2 * m + (V + 32) * E32 + 4 * E32 * z.abs().amax(1)
    f = (torch.ones(T) if weight is None else weight.cpu()).double() * has / tau
    full = torch.zeros((T, V), dtype=torch.float64).scatter_add_(1, at, q)
    named = torch.zeros((T, V)).scatter_add_(1, at, keep.float()) > 0
    dx = f[:, None] * ((p - full) @ w)
    wa = w.abs()
    db = 1.05 * (f.abs()[:, None] * (torch.where(named, 0.0, p) @ wa * u + r[:, None] * (p @ wa) + (k + 12) * E32 * ((p + full) @ wa))
                 + u * dx.abs()) + 1e-30
    return (loss, lb), (dx, db)


def check(got, want, name):
    value, bound = want
    got = got.detach().cpu().double()
    ok = (got - value).abs() <= bound
    assert bool(ok.all()), "%s: %d of %d elements off, the worst by %.3g times its bound" % (
        name, int((~ok).sum()), ok.numel(), float(((got - value).abs() / bound).nan_to_num(nan=math.inf).max()))


def make(T, K, V, k, dtype, seed=0, std=2.0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn((V, K), generator=g) * std / math.sqrt(K)).to(dtype)
    ids = torch.randint(V, (T, k), generator=g, dtype=torch.int32)  # some come twice
    X = torch.randn((T, K), generator=g) + 2.0 * W[ids[:, 0].long()].float()
    teacher = 3 * torch.randn((T, k), generator=g)
    weight = torch.rand((T,), generator=g) - 0.3
    return X.to(dtype).cuda(), W.cuda(), ids.cuda(), teacher.cuda(), weight.cuda()


def run(X, W, ids, teacher, tau, weight, Wt=None, dX=None):
    from paper_2607_28848_amd import vocab
    loss_w, dx_w = oracle(X, W, ids, teacher, tau, weight)
    alone = vocab.distill(X, W, ids, teacher, temperature=tau)
    loss, dx = vocab.distill_grad(X, W, ids, teacher, temperature=tau, weight=weight, Wt=Wt, dX=dX)
    torch.cuda.synchronize()
    check(alone, loss_w, "loss alone")
    check(loss, loss_w, "loss")
    check(dx, dx_w, "dX")
    return loss, dx


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,K,V,k,tau", [(1, 64, 1000, 1, 1.0), (5, 8, 7, 5, 2.0), (3, 72, 1, 3, 1.0), (128, 64, 256, 17, 0.5),
                                         (129, 520, 255, 64, 1.0), (333, 512, 5003, 13, 3.5), (64, 128, 8, 4, 1.0), (300, 264, 1032, 65, 2.0),
                                         (1, 4096, 20000, 100, 1.0), (513, 72, 2049, 7, 1.0), (2, 1000, 511, 1024, 1.0), (9, 64, 3000, 300, 4.0)])
def test_shapes(dtype, T, K, V, k, tau):
    print(dtype, T, K, V, k, tau, flush=True)
    X, W, ids, teacher, weight = make(T, K, V, k, dtype)
    _, a = run(X, W, ids, teacher, tau, weight)
    _, b = run(X, W, ids, teacher, tau, weight, Wt=W.t().contiguous())
    if V % 8 or dtype == F32:
        assert torch.equal(a, b)  # the transposed head is not read


@pytest.mark.parametrize("dtype", [BF, F32])
def test_padding_and_masked_entries(dtype):
    """Ids outside the vocabulary are no entries whatever their logits; rows of none, or of -infinity alone, are zeros."""
    from paper_2607_28848_amd import vocab
    X, W, ids, teacher, weight = make(150, 64, 777, 9, dtype, seed=3)
    for i, bad in ((0, -1), (17, 777), (18, -(1 << 31)), (149, (1 << 31) - 1)):
        ids[i, 2:] = bad
        teacher[i, 2:] = math.nan
    teacher[30, 1:4] = -math.inf
    none = (5, 40, 41)
    ids[5] = -1
    teacher[40] = -math.inf
    ids[41, :5], teacher[41, 5:] = 777, -math.inf
    X[5] = math.nan
    loss, dx = run(X, W, ids, teacher, 1.5, weight)
    for i in none:
        assert float(loss[i]) == 0.0 and bool((dx[i] == 0).all())
    # the other rows are what they are without those rows' values
    X[40] = math.inf
    again = vocab.distill_grad(X, W, ids, teacher, temperature=1.5, weight=weight)
    assert torch.equal(again[0], loss) and torch.equal(again[1], dx)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_entry_is_the_cross_entropy(dtype):
    """All entries at one token: the vocabulary loss against it and, being three entries of sum 1, sum_j q_j log q_j, since
    sum_j q_j (log q_j - log p) = sum_j q_j log q_j - log p; the same gradient.  One entry: q = 1, the loss itself."""
    from paper_2607_28848_amd import vocab
    X, W, ids, teacher, weight = make(140, 64, 777, 3, dtype, seed=4)
    ids[:] = ids[:, :1]
    loss, dx = run(X, W, ids, teacher, 1.0, weight)
    one, one_dx = run(X, W, ids[:, :1].contiguous(), teacher[:, :1].contiguous(), 1.0, weight)
    want, want_dx = vocab.loss_grad(X, W, ids[:, 0].contiguous(), weight=weight)
    (_, lb), (_, db) = oracle(X, W, ids, teacher, 1.0, weight)
    q = torch.softmax(teacher.cpu().double(), 1)
    # either side within its bound
    both = 2 * lb + 2 * E32 * want.cpu().double().abs()
    off = (loss.double() - want.double()).cpu() - (q * torch.log(q)).sum(1)
    assert float((off.abs() - both).max()) <= 0 and float(((one.double() - want.double()).cpu().abs() - both).max()) <= 0
    for x in (dx, one_dx):
        assert float(((x.double() - want_dx.double()).cpu().abs() - 2 * db).max()) <= 0


def test_agreement_keeps_its_accuracy():
    """bf16: a teacher that is the student itself (all of a small vocabulary): the gradient is a difference of equal
    terms, of which none is rounded to bf16."""
    from paper_2607_28848_amd import vocab
    g = torch.Generator().manual_seed(1)
    T, K, V = 40, 256, 200
    W = (torch.randn((V, K), generator=g) * 2 / 16).to(BF).cuda()
    X = torch.randn((T, K), generator=g).to(BF).cuda()
    ids = torch.arange(V, dtype=torch.int32).expand(T, V).contiguous().cuda()
    teacher = (X.double() @ W.double().t()).float()
    loss, dx = run(X, W, ids, teacher, 1.0, None)
    p = torch.softmax(teacher.double(), 1)
    z = teacher.double().abs().amax()
    # the teacher's logits are rounded to fp32, the student's to fp32 of K products; shares once: see the bounds above
    assert float(loss.abs().max()) <= (2 * (K + 4) * 2 * float((X.abs().double() @ W.abs().double().t()).max()) + V + 40) * E32
    bound = (p @ W.abs().double()) * (2 * (K + 4) * float((X.abs().double() @ W.abs().double().t()).max()) + 2 * V + 50 + 8 * float(z)) * E32
    assert bool((dx.double().abs() <= bound * 1.01).all())


def test_sure_students_in_fp32():
    """Rows whose mass is at their entries' tokens: those terms are not the products' (whose K-long fp32 sums err by up to
    m) but formed apart, so m bounds the other terms alone; 64 e and 8 e of the loss are left for sums and logarithms.  The
    losses alone and those beside the gradient are the same bits."""
    from paper_2607_28848_amd import vocab
    T, K, V, k = 50, 1024, 3000, 6
    X, W, ids, teacher, _ = make(T, K, V, k, F32, seed=12)
    X += 3.0 * W[ids[:, 0].long()] + 2.0 * W[ids[:, 1].long()]
    loss = vocab.distill(X, W, ids, teacher)
    again, _ = vocab.distill_grad(X, W, ids, teacher)
    torch.cuda.synchronize()
    assert torch.equal(loss, again)
    (want, _), _ = oracle(X, W, ids, teacher, 1.0, None)
    z = X.cpu().double() @ W.cpu().double().t()
    p = torch.softmax(z, 1)
    rest = 1 - torch.zeros_like(p).scatter(1, ids.cpu().long(), 1.0).mul(p).sum(1)
    m = ((K + 4) * (X.abs().cpu().double() @ W.abs().cpu().double().t()) + 4 * z.abs()).amax(1) * E32
    assert float(rest.median()) < 0.2
    bound = 1.05 * (rest * (2 * m + (V + 40) * E32) + (64 + 8 * want.abs()) * E32)
    # what 8 products in fp32 leave of an entry's own logit
    bound += 8 * E32 * (X.abs().cpu().double() @ W.abs().cpu().double().t()).gather(1, ids.cpu().long()).amax(1) / 8
    off = (loss.cpu().double() - want).abs()
    assert float((off / bound).max()) <= 1, float((off / bound).max())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("std", [1e-3, 40.0])
def test_flat_and_sure_students(dtype, std):
    """Logits of thousandths, and of hundreds, whose references differ from tile to tile."""
    X, W, ids, teacher, weight = make(70, 128, 3000, 12, dtype, seed=5, std=std)
    run(X, W, ids, teacher, 1.0, weight)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pieces_of_the_vocabulary(dtype):
    """More columns than a piece's room: entries in the first, a middle and the last piece, and at their borders."""
    from paper_2607_28848_amd import vocab
    T, K, V, k = (900, 64, 400000, 6) if dtype == BF else (900, 64, 200000, 6)
    g = torch.Generator(device="cuda").manual_seed(6)
    W = (torch.randn((V, K), generator=g, device="cuda") * 0.25).to(dtype)
    X = torch.randn((T, K), generator=g, device="cuda").to(dtype)
    ids = torch.randint(V, (T, k), generator=g, device="cuda", dtype=torch.int32)
    width = (256 << 20) // (2 if dtype == BF else 4) // T
    assert width < V / 2
    ids[0] = torch.tensor([0, V - 1, width, width - 1, width // 256 * 256, width // 256 * 256 - 1], dtype=torch.int32)
    teacher = 3 * torch.randn((T, k), generator=g, device="cuda")
    loss, dx = vocab.distill_grad(X, W, ids, teacher, temperature=2.0)
    alone = vocab.distill(X, W, ids, teacher, temperature=2.0)
    rows = torch.cat((torch.arange(3), torch.arange(T - 3, T))).cuda()
    loss_w, dx_w = oracle(X[rows], W, ids[rows], teacher[rows], 2.0, None)
    check(loss[rows], loss_w, "loss")
    check(alone[rows], loss_w, "loss alone")
    check(dx[rows], dx_w, "dX")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_and_ends(dtype):
    """Rows further apart than they are long; what lies around the outputs stays."""
    from paper_2607_28848_amd import vocab
    T, K, V, k = 37, 72, 515, 5
    X, W, ids, teacher, weight = make(T, K, V, k, dtype, seed=7)

    def strided(t, ld):
        b = torch.full((t.shape[0], ld), math.nan, dtype=t.dtype, device="cuda")
        b[:, :t.shape[1]] = t
        return b[:, :t.shape[1]]

    room = torch.full((T + 2, K + 24), 7.0, dtype=dtype, device="cuda")
    dX, loss = room[1:-1, 8:8 + K], torch.full((T + 2,), 7.0, device="cuda")
    Wt = strided(W.t().contiguous(), V + 5)
    vocab.distill_grad(strided(X, K + 16), strided(W, K + 8), ids, teacher, temperature=1.0, weight=weight, Wt=Wt, dX=dX,
                       loss=loss[1:-1])
    torch.cuda.synchronize()
    loss_w, dx_w = oracle(X, W, ids, teacher, 1.0, weight)
    check(loss[1:-1], loss_w, "loss")
    check(dX, dx_w, "dX")
    room[1:-1, 8:8 + K] = 7.0
    assert bool((room == 7).all()) and float(loss[0]) == float(loss[-1]) == 7.0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_logits(dtype):
    """A logit of -infinity drops out of the sums; one of NaN or infinity at any token reaches the losses of its rows."""
    from paper_2607_28848_amd import vocab
    X, W, ids, teacher, weight = make(20, 64, 300, 4, dtype, seed=11)
    ids %= 200
    X[:, 0] = 1.0
    W[250, 0] = -math.inf
    W0 = W.clone()
    W0[250] = 0
    W0[250, 0] = -3e4  # exp of it is 0
    loss, dx = vocab.distill_grad(X, W, ids, teacher, weight=weight)
    want, want_dx = vocab.distill_grad(X, W0, ids, teacher, weight=weight)
    assert torch.equal(loss, want) and torch.equal(dx[:, 1:], want_dx[:, 1:])
    assert torch.equal(vocab.distill(X, W, ids, teacher), vocab.distill(X, W0, ids, teacher))
    for bad in (math.inf, math.nan):
        W[250, 0] = bad
        loss, _ = vocab.distill_grad(X, W, ids, teacher, weight=weight)
        assert not bool(loss.isfinite().any()) and not bool(vocab.distill(X, W, ids, teacher).isfinite().any())
    # at an entry's own token: log p of it is -infinity
    W[250] = W0[10]
    W[10, 0] = -math.inf
    ids[:], ids[3, 1] = ids % 10, 10
    loss, _ = vocab.distill_grad(X, W, ids, teacher, weight=weight)
    ok = torch.ones(20, dtype=torch.bool)
    ok[3] = False
    assert float(loss[3]) == math.inf and bool(loss.cpu()[ok].isfinite().all())


def test_no_rows():
    from paper_2607_28848_amd import vocab
    W = torch.randn((50, 64), device="cuda")
    X, ids, t = torch.empty((0, 64), device="cuda"), torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 4), device="cuda")
    loss, dx = vocab.distill_grad(X, W, ids, t)
    assert loss.shape == (0,) and dx.shape == (0, 64) and vocab.distill(X, W, ids, t).shape == (0,)


def test_streams_and_graph_replays():
    """The same bits from call to call and on another stream; a captured pass replayed on new inputs."""
    from paper_2607_28848_amd import vocab
    T, K, V, k = 200, 264, 3001, 11
    X, W, ids, teacher, weight = make(T, K, V, k, BF, seed=8)

    def eager(stream=None):
        return vocab.distill_grad(X, W, ids, teacher, temperature=2.0, weight=weight, stream=stream)

    first = eager()
    torch.cuda.synchronize()
    for out in (eager(), eager(torch.cuda.Stream())):
        torch.cuda.synchronize()
        assert torch.equal(first[0], out[0]) and torch.equal(first[1], out[1])
    ws = torch.empty(vocab.distill_workspace_bytes(T, K, V, k, BF, True), dtype=torch.uint8, device="cuda")
    loss, dX = torch.empty_like(first[0]), torch.empty_like(first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vocab.distill_grad(X, W, ids, teacher, temperature=2.0, weight=weight, loss=loss, dX=dX, workspace=ws)
    for seed in range(3):
        x, _, i, t, w = make(T, K, V, k, BF, seed=20 + seed)
        for to, new in ((X, x), (ids, i), (teacher, t), (weight, w)):
            to.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(dX, want[1])


def test_gradient_against_differences():
    """fp32: the directional derivative of the weighted losses' sum by central differences: third order, 8 h^2 of the terms."""
    from paper_2607_28848_amd import vocab
    X, W, ids, teacher, weight = make(30, 64, 400, 7, F32, seed=9)
    _, dx = vocab.distill_grad(X, W, ids, teacher, temperature=1.5, weight=weight)
    u = torch.randn(X.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    h = 2.0 ** -6

    def L(x):
        return float((vocab.distill(x, W, ids, teacher, temperature=1.5).double() * weight.double()).sum())

    num = (L(X + h * u) - L(X - h * u)) / (2 * h)
    terms = dx.double() * u.double()
    # rounding of the losses, 30 of about 5, over 2 h
    assert abs(num - float(terms.sum())) <= 8 * h * h * float(terms.abs().sum()) + 30 * 8 * 600 * E32 / (2 * h)
