"""The vocabulary loss on the GPU against the definition in 64 bits: odd rows and vocabularies, several pieces, moving
references, rows without a target, strides, and the gradient against differences.

Bounds are first-order worst cases.  u is 2^-8 in bf16 (8 significant bits) and 2^-24 in fp32, e = 2^-24.  A logit's
error is at most ez = (K + 4) e sum|x||w|; with m the row's largest ez, a probability's relative error is at most
r = 2 m + (V + 32) e, and that of a term as an operand u more.  The loss is log(1 + (1 - p_t) / p_t), so (1 - p_t) r
bounds what the sums bring, and 16 e (|loss| + |ref|) the final logarithm where p_t is below a half.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E32 = 2.0 ** -24


def oracle(X, W, target, weight):
    u = 2.0 ** -8 if X.dtype == BF else E32
    x, w = X.detach().cpu().double(), W.detach().cpu().double()
    T, K = x.shape
    V = w.shape[0]
    t = target.cpu().long()
    has = (t >= 0) & (t < V)
    x = torch.where(has[:, None], x, 0.0)
    at = torch.where(has, t, 0)[:, None]
    z = x @ w.t()
    m = ((K + 4) * E32 * (x.abs() @ w.abs().t())).amax(dim=1)
    lse = torch.logsumexp(z, dim=1)
    p = torch.exp(z - lse[:, None])
    loss = torch.where(has, lse - z.gather(1, at)[:, 0], 0.0)
    q = p.scatter(1, at, 0.0)            # the terms that are not the target's
    rest = q.sum(dim=1)
    r = 2 * m + (V + 32) * E32
    # log1p where p_t is above a half: lse - z_t cancels in the oracle itself
    loss = torch.where(has & (rest < 0.5), torch.log1p(rest / p.gather(1, at)[:, 0]), loss)
    lb = 1.05 * (rest * r + 16 * E32 * (loss.abs() + torch.where(rest >= 0.5, z.abs().amax(dim=1), 0.0))) * has + 1e-30
    f = (torch.ones(T) if weight is None else weight.cpu()).double() * has
    wt = w[at[:, 0]]
    dx = f[:, None] * (q @ w - rest[:, None] * wt)
    db = 1.05 * (f.abs()[:, None] * ((u + r)[:, None] * (q @ w.abs()) + (rest * r)[:, None] * wt.abs() +
                                     8 * E32 * (q @ w.abs() + rest[:, None] * wt.abs())) + u * dx.abs()) + 1e-30
    return (loss, lb), (dx, db)


def check(got, want, name):
    value, bound = want
    got = got.detach().cpu().double()
    ok = (got - value).abs() <= bound
    assert bool(ok.all()), "%s: %d of %d elements off, the worst by %.3g times its bound" % (
        name, int((~ok).sum()), ok.numel(), float(((got - value).abs() / bound).nan_to_num(nan=math.inf).max()))


def strided(t, ld):
    b = torch.full((t.shape[0], ld), math.nan, dtype=t.dtype, device="cuda")
    b[:, :t.shape[1]] = t
    return b[:, :t.shape[1]]


def make(T, K, V, dtype, seed=0, std=2.0, lean=True):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn((V, K), generator=g) * std / math.sqrt(K)).to(dtype)
    target = torch.randint(V, (T,), generator=g, dtype=torch.int32)
    X = torch.randn((T, K), generator=g)
    if lean:
        X += (torch.rand((T, 1), generator=g) < 0.5) * 3.0 * W[target.long()].float()
    weight = torch.rand((T,), generator=g) - 0.3
    return X.to(dtype).cuda(), W.cuda(), target.cuda(), weight.cuda()


def run(X, W, target, weight, Wt=None, dX=None):
    from paper_2607_28848_amd import vocab
    (loss_w, dx_w) = oracle(X, W, target, weight)
    check(vocab.loss(X, W, target), loss_w, "loss alone")
    loss, dx = vocab.loss_grad(X, W, target, weight=weight, Wt=Wt, dX=dX)
    check(loss, loss_w, "loss")
    check(dx, dx_w, "dX")
    return loss, dx


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,K,V", [(1, 64, 1000), (5, 8, 7), (3, 72, 1), (128, 64, 256), (129, 520, 255), (333, 512, 5003),
                                   (64, 128, 8), (300, 264, 1032), (1, 4096, 20000), (513, 72, 2049), (2, 1000, 511)])
def test_shapes(dtype, T, K, V):
    print(dtype, T, K, V, flush=True)
    X, W, target, weight = make(T, K, V, dtype)
    _, a = run(X, W, target, weight)
    _, b = run(X, W, target, weight, Wt=W.t().contiguous())
    if V % 8 or dtype == F32:
        assert torch.equal(a, b)  # the transposed head is not read


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_without_a_target(dtype):
    """Losses and gradients of such rows are zeros, whatever they hold; the others are what they are without them."""
    from paper_2607_28848_amd import vocab
    X, W, target, weight = make(140, 64, 777, dtype, seed=3)
    for i, t in ((0, -1), (17, 777), (18, -100), (139, 2 ** 31 - 1), (100, -2 ** 31)):
        target[i] = t
    X[17] = math.nan
    X[100] = math.inf
    loss, dx = run(X, W, target, weight)
    gone = [0, 17, 18, 139, 100]
    assert bool((loss[gone] == 0).all()) and bool((dx[gone] == 0).all())
    loss, dx = vocab.loss_grad(X, W, torch.full_like(target, -1))
    assert bool((loss == 0).all()) and bool((dx == 0).all())
    loss, dx = vocab.loss_grad(X[:0], W, target[:0])
    assert loss.shape == (0,) and dx.shape == (0, 64)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides(dtype):
    """Rows further apart than they are long: the same bits, and nothing between the rows is touched."""
    T, K, V = 150, 136, 1000
    X, W, target, weight = make(T, K, V, dtype, seed=5)
    Wt = W.t().contiguous()
    a = run(X, W, target, weight, Wt=Wt)
    dX = strided(torch.zeros((T, K), dtype=dtype, device="cuda"), K + 24)
    b = run(strided(X, K + 8), strided(W, K + 64), target, weight, Wt=strided(Wt, V + 40), dX=dX)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bool(dX._base[:, K:].isnan().all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rise", [0.0, 30.0])
def test_pieces(dtype, rise):
    """Head rows 2^20 elements apart leave room for 512 columns a piece: three of them, with Wt and without; with
    `rise`, every 300 columns' logits lie above the ones before by more than what leaves a reference where it is."""
    T, K, V = 200, 64, 1200
    X, W, target, weight = make(T, K, V, dtype, seed=7)
    X[:, 0] = 1.0
    W[:, 0] = (rise * (torch.arange(V, device="cuda") // 300)).to(dtype)
    a = run(X, strided(W, 1 << 20), target, weight)
    b = run(X, strided(W, 1 << 20), target, weight, Wt=W.t().contiguous())
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sure_and_impossible_targets(dtype):
    """Losses from 1e-12 to hundreds keep their accuracy, and so do their gradients; logits of -infinity drop out."""
    K, V = 64, 300
    X, W, _, _ = make(40, K, V, dtype, seed=9, std=0.2)
    X[:, 0] = torch.linspace(-30, 30, 40, device="cuda").to(dtype)
    W[:, 0] = 0
    W[5, 0] = 8.0
    target = torch.full((40,), 5, dtype=torch.int32, device="cuda")
    run(X, W, target, None)


def test_repeats_streams_and_graphs():
    from paper_2607_28848_amd import vocab
    T, K, V = 300, 256, 4000
    X, W, target, weight = make(T, K, V, BF, seed=11)
    ws = torch.empty(vocab.workspace_bytes(T, K, V, BF, grad=True), dtype=torch.uint8, device="cuda")
    loss, dx = (t.clone() for t in vocab.loss_grad(X, W, target, weight=weight, workspace=ws))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        l2, d2 = vocab.loss_grad(X, W, target, weight=weight)
    torch.cuda.synchronize()
    assert torch.equal(loss, l2) and torch.equal(dx, d2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vocab.loss_grad(X, W, target, weight=weight, loss=l2, dX=d2, workspace=ws)
    for seed in (11, 12, 13):
        X2, _, t2, w2 = make(T, K, V, BF, seed=seed)
        for t, b in ((X, X2), (target, t2), (weight, w2)):
            t.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        el, ed = vocab.loss_grad(X, W, target, weight=weight)
        torch.cuda.synchronize()
        assert torch.equal(l2, el) and torch.equal(d2, ed)


def test_gradient_against_differences():
    """fp32: the directional derivative of the weighted losses by central differences (third-order error)."""
    from paper_2607_28848_amd import vocab
    X, W, target, weight = make(70, 96, 500, F32, seed=13)
    u = torch.randn(X.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    _, dx = vocab.loss_grad(X, W, target, weight=weight)
    h = 2.0 ** -6

    def L(x):
        return float((vocab.loss(x, W, target).double() * weight.double()).sum())

    num = (L(X + h * u) - L(X - h * u)) / (2 * h)
    terms = dx.double() * u.double()
    assert abs(num - float(terms.sum())) <= 8 * h * h * float(terms.abs().sum())


def test_refusals():
    from paper_2607_28848_amd import dsv, vocab
    lib = dsv.lib_handle()
    X, W, target, weight = make(10, 64, 100, BF)
    ws = torch.empty(vocab.workspace_bytes(10, 64, 100, BF, grad=True), dtype=torch.uint8, device="cuda")
    dx, loss = torch.zeros_like(X), torch.zeros(10, device="cuda")
    p = dict(dt=0, T=10, K=64, V=100, X=X.data_ptr(), ldx=0, W=W.data_ptr(), ldw=0, Wt=None, ldwt=0, t=target.data_ptr(),
             w=weight.data_ptr(), l=loss.data_ptr(), dx=dx.data_ptr(), lddx=0, ws=ws.data_ptr(), n=ws.numel())

    def call(**kw):
        q = dict(p, **kw)
        return lib.dsv_vocab_loss_grad(q["dt"], q["T"], q["K"], q["V"], q["X"], q["ldx"], q["W"], q["ldw"], q["Wt"],
                                       q["ldwt"], q["t"], q["w"], q["l"], q["dx"], q["lddx"], q["ws"], q["n"], None)

    for kw, want in ((dict(T=-1), dsv.ERR_ARG), (dict(X=None), dsv.ERR_ARG), (dict(W=p["W"] + 2), dsv.ERR_ARG),
                     (dict(t=None), dsv.ERR_ARG), (dict(w=p["w"] + 1), dsv.ERR_ARG), (dict(l=p["l"] + 2), dsv.ERR_ARG),
                     (dict(dx=None), dsv.ERR_ARG), (dict(ws=None), dsv.ERR_ARG), (dict(ws=p["ws"] + 16), dsv.ERR_ARG),
                     (dict(dt=3), dsv.ERR_RANGE), (dict(K=60), dsv.ERR_SIZE), (dict(K=0), dsv.ERR_SIZE),
                     (dict(V=0), dsv.ERR_SIZE), (dict(V=(1 << 24) + 1), dsv.ERR_SIZE), (dict(ldx=56), dsv.ERR_SIZE),
                     (dict(ldw=68), dsv.ERR_SIZE), (dict(lddx=1 << 21), dsv.ERR_SIZE), (dict(n=p["n"] - 1), dsv.ERR_SIZE),
                     (dict(l=None), dsv.OK), (dict(w=None), dsv.OK)):
        assert call(**kw) == want, kw
    for bad in (dict(X=X.half()), dict(W=W.float()), dict(target=target.long()), dict(weight=weight[:9]),
                dict(Wt=W), dict(dX=dx[:9])):
        a = dict(dict(X=X, W=W, target=target, weight=weight, Wt=None, dX=dx), **bad)
        with pytest.raises((TypeError, ValueError)):
            vocab.loss_grad(**a)
    torch.cuda.synchronize()
