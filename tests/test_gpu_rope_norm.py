"""How exact the norm is in fp32, where nothing but its inverse root and two products is rounded.

Elements are whole numbers up to 63, so their squares' sum is exact in fp32 in any order, as is the mean (a quotient by 64 or
128); eps = 2^-100 is lost in it and changes the value by less.  The weight is 1.  With e = 2^-24 the inverse root is rounded
once: what comes before its last step is right to 6 e^2 (the step squares an error of 2 e) and the step's correction, of 2 e,
to 2 e of itself.  Times x is one rounding more, times 1 none: 2 e (1 + 8 e) of each element, below 2.001 e.  (The instruction
for inverse roots alone, good to a whole unit in the last place, leaves elements off by 2.06 e.)  Backward an upstream gradient of
one element is taken, so that nothing cancels: at the others dx = -r x_i (x_j r) r g / d."""
import pytest
import torch

pytestmark = pytest.mark.gpu
E32 = 2.0 ** -24


def make(d, n=4000):
    gen = torch.Generator().manual_seed(d)
    x = torch.randint(-63, 64, (n, 3, d), generator=gen).float()
    x[:, :, 0] = 63  # no vector is 0
    return x, torch.rsqrt((x.double() ** 2).mean(-1, keepdim=True))


@pytest.mark.parametrize("d", [64, 128])
def test_forward(d):
    from paper_2607_28848_amd import rope
    x, r = make(d)
    w = torch.ones(d, device="cuda")
    y, _ = rope.fwd(x.cuda(), None, None, None, q_weight=w, eps=2.0 ** -100)
    torch.cuda.synchronize()
    want = x.double() * r
    off = (y.cpu().double() - want).abs()
    assert bool((off <= 2.001 * E32 * want.abs()).all()), float((off / (E32 * want.abs()).clamp_min(1e-30)).max())


@pytest.mark.parametrize("d", [64, 128])
def test_backward(d):
    """dx_i = -r^3 x_i x_0 / d at i > 0 for a gradient of 1 at element 0: three roots (e each), the products x_0 r, x_i r, times
    the mean of one product (the other summands are 0), and times r: 7 e, and e for the difference from 0: 8 e."""
    from paper_2607_28848_amd import rope
    x, r = make(d)
    w, g = torch.ones(d, device="cuda"), torch.zeros_like(x)
    g[:, :, 0] = 1
    dx, _, dw, _ = rope.bwd(g.cuda(), None, None, None, Q=x.cuda(), q_weight=w, eps=2.0 ** -100)
    torch.cuda.synchronize()
    want = -(r ** 3) * x.double() * x[:, :, :1].double() / d
    off = (dx.cpu().double() - want).abs()[:, :, 1:]
    assert bool((off <= 8.001 * E32 * want.abs()[:, :, 1:]).all()), float((off / (E32 * want.abs()[:, :, 1:]).clamp_min(1e-30)).max())
    # the weight's gradient: 12000 positive terms of 63 r, in sums of rows' chains and of 64 bits
    total = (63 * r).sum()
    assert abs(float(dw[0].cpu().double() - total)) <= (4000 + 8) * E32 * float(total) and bool((dw[1:] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_ends_of_the_range(dtype):
    """An eps that is the smallest normal number under zeros; an infinite element among finite ones; a mean square past fp32."""
    from paper_2607_28848_amd import rope
    x = torch.zeros((3, 1, 64), dtype=dtype, device="cuda")
    x[1, 0, 5] = float("inf")
    x[1, 0, 6] = 2.0
    x[2] = 2.0 ** 100
    y, _ = rope.fwd(x, None, None, None, q_weight=torch.ones(64, device="cuda"), eps=2.0 ** -126)
    torch.cuda.synchronize()
    y = y.cpu()[:, 0]
    assert bool((y[0] == 0).all()) and bool((y[2] == 0).all())
    assert bool(y[1, 5].isnan()) and bool((y[1, :5] == 0).all()) and bool((y[1, 6:] == 0).all())
