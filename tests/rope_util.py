"""The oracle of the norms and the position rotation: 64 bits on the CPU, gradients by autograd of the plain formula, with
a bound on what a kernel of the given type may be off, element by element.

u is the unit roundoff of the output's one rounding (2^-8 for bf16, 2^-24 for fp32), e = 2^-24 that of fp32 steps.  A norm's
mean square is a sum of positive terms, 16 a lane and 3 joins, off by at most 20 e of itself, so its inverse root by 10 e
and 2 e of its own; times x and w: 15 e.  A cosine or sine is off by at most 5 e: the reduced angle's rounding, the series'
steps.  A turned pair adds three steps.  So an output is off by at most u |y| + 24 e (|u_a| + |u_b|).
"""
import torch

E32 = 2.0 ** -24


def unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else E32


def pairs(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def formula(x, pos, freq, weight, eps, interleaved):
    """[rows][heads][d] in 64 bits, and |u_a| + |u_b| of each element's pair (an unturned one: |u|)."""
    u = x
    if weight is not None:
        u = x * weight / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if freq is None:
        return u, u.abs()
    a, b = pairs(2 * len(freq), interleaved)
    angle = (pos.double()[:, None] * freq[None, :])[:, None, :]
    y, size = u.clone(), u.detach().abs().clone()
    y[..., a] = u[..., a] * torch.cos(angle) - u[..., b] * torch.sin(angle)
    y[..., b] = u[..., b] * torch.cos(angle) + u[..., a] * torch.sin(angle)
    both = u.detach()[..., a].abs() + u.detach()[..., b].abs()
    size[..., a], size[..., b] = both, both
    return y, size


def forward(x, pos, freq, weight, eps, interleaved, dtype):
    """(value, bound)"""
    x, pos, freq, weight = (None if t is None else t.detach().cpu() for t in (x, pos, freq, weight))
    y, size = formula(x.double(), pos, freq, None if weight is None else weight.double(), eps, interleaved)
    return y, unit(dtype) * y.abs() + 24 * E32 * size


def backward(dy, x, pos, freq, weight, eps, interleaved, dtype):
    """((dx, bound), (dw, bound)) of gradient rows dy; x and pos are those rows' own."""
    dy, x, pos, freq, weight = (None if t is None else t.detach().cpu() for t in (dy, x, pos, freq, weight))
    dy = dy.double()
    x = torch.ones_like(dy) if x is None else x.double()
    x.requires_grad_(True)
    w = None if weight is None else weight.double().requires_grad_(True)
    y, _ = formula(x, pos, freq, w, eps, interleaved)
    grads = torch.autograd.grad(y, [x] if w is None else [x, w], dy)
    dx = grads[0]
    # the gradient turned back, and the pair's absolute sum
    g, size = formula(dy, None if pos is None else -pos.double(), freq, None, eps, interleaved)
    if w is None:
        return (dx, unit(dtype) * dx.abs() + 24 * E32 * size), None
    x = x.detach()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    wa = weight.double().abs()
    # terms: r g w and r xhat mean(g w xhat); 15 e from xhat and r on either side, 8 e from g, 20 e from the mean
    terms = r * (size * wa + (x * r).abs() * (size * wa * (x * r).abs()).mean(-1, keepdim=True))
    n_rows, heads = dy.shape[0], dy.shape[1]
    chain = n_rows * ((heads + 7) // 8) + 64  # a lane has a head of every eight, or of more
    dwb = (chain + 40) * E32 * (size * (x * r).abs()).sum((0, 1)) + E32 * grads[1].abs()
    return (dx, unit(dtype) * dx.abs() + 64 * E32 * terms), (grads[1], dwb)
