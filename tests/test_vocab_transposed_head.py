"""Which transposed heads the vocabulary loss reads: its tiles address 256 rows of one in 31 bits.  On the CPU, without
rows nothing is launched, and a transposed head that would be read is refused for its alignment."""
import pytest
import torch

from paper_2607_28848_amd import dsv

BUF = 1 << 30  # an address that nothing reads


def refused(V, ldwt=0, dt=dsv.BF16):
    return dsv.lib_handle().dsv_vocab_loss_grad(dt, 0, 64, V, BUF, 0, BUF, 0, BUF + 2, ldwt, BUF, None, BUF, BUF, 0, BUF,
                                                1 << 40, None)


@pytest.mark.parametrize("V,ldwt,want", [
    (8, 0, dsv.ERR_ARG), (1 << 20, 0, dsv.ERR_ARG), (1 << 20, 1 << 20, dsv.ERR_ARG), ((1 << 22) - 8, 0, dsv.ERR_ARG),
    (1 << 22, 0, dsv.OK), ((1 << 22) + 8, 0, dsv.OK), (8421504, 0, dsv.OK), (1 << 24, 0, dsv.OK),  # read as the head lies
    (12, 0, dsv.OK), (8, (1 << 20) + 8, dsv.ERR_SIZE), (1 << 22, 1 << 22, dsv.ERR_SIZE)])
def test_transposed_heads_that_are_read(V, ldwt, want):
    assert refused(V, ldwt) == want
    assert refused(V, ldwt, dsv.F32) == dsv.OK


@pytest.mark.gpu
@pytest.mark.parametrize("V", [(1 << 22) - 8, (1 << 22) + 8])
def test_wide_heads(V):
    """dX on both sides of the limit.  Every column of the head has a mean of its own, which is what a row that is left
    out or taken for another one would miss.  Relative to the terms' sizes, a probability is off by the logits' errors
    (twice (K + 4) e sum|x||w|), its rounding and its sum's; no sum is a chain of more than V / 16 + 64 additions."""
    from paper_2607_28848_amd import vocab
    T, K, e, u = 2, 264, 2.0 ** -24, 2.0 ** -8
    g = torch.Generator(device="cuda").manual_seed(V)
    mean = (torch.arange(K, device="cuda") * 37 % 101 + 20) / 50.0
    W = (torch.randn((V, K), generator=g, device="cuda") * 0.1 + mean).bfloat16()
    X = (torch.randn((T, K), generator=g, device="cuda") * 0.5).bfloat16()
    target = torch.tensor([3, V - 1], dtype=torch.int32, device="cuda")
    loss, dx = vocab.loss_grad(X, W, target, Wt=W.t().contiguous())
    plain, dx0 = vocab.loss_grad(X, W, target)
    assert torch.equal(loss, plain)
    w, x = W.double(), X.double()
    z = x @ w.t()
    r = 2 * (K + 4) * e * (x.abs() @ w.abs().t()).amax(dim=1) + (V / 16 + 64) * e
    q = torch.softmax(z, dim=1)
    q[torch.arange(T), target.long()] = 0
    rest, wt = q.sum(dim=1, keepdim=True), w[target.long()]
    want = q @ w - rest * wt
    bound = 1.05 * ((u + r)[:, None] * (q @ w.abs()) + r[:, None] * rest * wt.abs() + u * want.abs())
    for got in (dx, dx0):
        assert bool(((got.double() - want).abs() <= bound).all()), float(((got.double() - want).abs() / bound).max())
