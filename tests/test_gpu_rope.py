"""Norms and the position rotation on the GPU against the 64-bit oracle: head counts and widths, partial and interleaved
rotations, one row to thousands, slots, strided and in-place tensors, far positions, gradients, streams and graphs."""
import math

import pytest
import torch

from attn_util import check
from rope_util import backward, forward

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def columns(n, hq, hkv, d, dtype, layout, gen):
    """q, k, v as a caller has them."""
    def normal(*s):
        return torch.randn(s, generator=gen)
    rows = (normal(n, hq + 2 * hkv, d) * torch.exp(normal(n, 1, 1))).to(dtype).cuda()
    if layout == "fused":
        return rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    q, k, v = (t.contiguous() for t in (rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]))
    if layout == "heads":
        return tuple(t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    def pad(t):  # rows and heads further apart than they are long
        b = torch.full((n, t.shape[1] + 1, d + 8), math.nan, dtype=dtype, device="cuda")
        b[:, :t.shape[1], :d] = t
        return b[:, :t.shape[1], :d]
    return pad(q), pad(k), pad(v)


def setting(n, d, rot, norm, gen, far=5000):
    pos = torch.randint(far, (n,), generator=gen, dtype=torch.int32).cuda()
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).cuda() if rot else None
    qw, kw = ((1 + 0.3 * torch.randn((d,), generator=gen)).cuda() if norm else None for _ in range(2))
    return pos, freq, qw, kw


SHAPES = [(32, 8, 128, 128, False, True, "fused"), (5, 1, 64, 64, True, True, "padded"), (8, 2, 128, 48, False, True, "heads"),
          (3, 3, 64, 16, True, False, "fused"), (16, 16, 64, 32, False, False, "padded"), (40, 1, 128, 0, False, True, "fused"),
          (7, 2, 128, 112, True, True, "heads")]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 9, 700])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dtype, n, shape):
    from paper_2607_28848_amd import rope
    hq, hkv, d, rot, nxt, norm, layout = shape
    print(dtype, n, shape, flush=True)
    gen = torch.Generator().manual_seed(n + hq)
    q, k, v = columns(n, hq, hkv, d, dtype, layout, gen)
    pos, freq, qw, kw = setting(n, d, rot, norm, gen)
    # slots in any order; some rows have none
    n_slots, mark = n + 5, 7.0
    slots = torch.randperm(n_slots, generator=gen)[:n].to(torch.int32)
    if n > 4:
        slots[1], slots[3], slots[4] = -1, n_slots, -(1 << 31)
    K, V = (torch.full((hkv, n_slots, d), mark, dtype=dtype, device="cuda").transpose(0, 1) for _ in range(2))
    Q, K2, V2 = rope.fwd(q, k, pos, freq, q_weight=qw, k_weight=kw, eps=EPS, interleaved=nxt, V=v, slots=slots.cuda(), K_out=K,
                         V_out=V)
    torch.cuda.synchronize()
    assert K2 is K and V2 is V
    check(Q, forward(q, pos, freq, qw, EPS, nxt, dtype), "Q")
    value, bound = forward(k, pos, freq, kw, EPS, nxt, dtype)
    kept = (slots >= 0) & (slots < n_slots)
    at = slots[kept].long()
    check(K.cpu()[at], (value[kept], bound[kept]), "K")
    assert torch.equal(V.cpu()[at], v.cpu()[kept])
    other = torch.ones(n_slots, dtype=torch.bool)
    other[at] = False
    assert bool((K.cpu()[other] == mark).all()) and bool((V.cpu()[other] == mark).all())
    # without slots, one tensor at a time: the same bits
    Q1, none = rope.fwd(q, None, pos, freq, q_weight=qw, eps=EPS, interleaved=nxt)
    none2, K1 = rope.fwd(None, k, pos, freq, k_weight=kw, eps=EPS, interleaved=nxt)
    torch.cuda.synchronize()
    assert none is None and none2 is None and torch.equal(Q1, Q) and torch.equal(K1.cpu()[kept], K.cpu()[at])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,shape", [(m, s) for s in SHAPES for m in (1, 2, 65, 513)] + [(5000, s) for s in SHAPES[1:4]])
def test_backward(dtype, m, shape):
    from paper_2607_28848_amd import rope
    hq, hkv, d, rot, nxt, norm, layout = shape
    print(dtype, m, shape, flush=True)
    n = m + 11
    gen = torch.Generator().manual_seed(m + hq)
    q, k, _ = columns(n, hq, hkv, d, dtype, layout, gen)
    pos, freq, qw, kw = setting(n, d, rot, norm, gen)
    rows = torch.randint(n, (m,), generator=gen, dtype=torch.int32)  # rows may come twice
    if m > 10:
        rows[3], rows[7] = -1, n
    dQ, dK, _ = columns(m, hq, hkv, d, dtype, layout, gen)
    out = rope.bwd(dQ, dK, pos, freq, rows=rows.cuda(), Q=q, K=k, q_weight=qw, k_weight=kw, eps=EPS, interleaved=nxt)
    torch.cuda.synchronize()
    assert (out[2] is None) == (not norm) and (out[3] is None) == (not norm)
    in_ = ((rows >= 0) & (rows < n))
    at = rows[in_].long()
    for name, dy, x, w, dx, dw in (("dQ", dQ, q, qw, out[0], out[2]), ("dK", dK, k, kw, out[1], out[3])):
        (value, bound), weight = backward(dy.cpu()[in_], x.cpu()[at], pos.cpu()[at], freq, w, EPS, nxt, dtype)
        check(dx.cpu()[in_], (value, bound), name)
        assert bool((dx.cpu()[~in_] == 0).all())
        if norm:
            check(dw, weight, name + " weight")
    again = rope.bwd(dQ, dK, pos, freq, rows=rows.cuda(), Q=q, K=k, q_weight=qw, k_weight=kw, eps=EPS, interleaved=nxt)
    # into given rows without the weights' gradients, and one tensor alone: the same bits
    a, b = torch.empty_like(out[0]), torch.empty_like(out[1])
    some = rope.bwd(dQ, dK, pos, freq, rows=rows.cuda(), Q=q, K=k, q_weight=qw, k_weight=kw, eps=EPS, interleaved=nxt, dQ_out=a,
                    dK_out=b)
    alone = rope.bwd(dQ, None, pos, freq, rows=rows.cuda(), Q=q, q_weight=qw, eps=EPS, interleaved=nxt)
    torch.cuda.synchronize()
    assert some[2] is None and some[3] is None and alone[1] is None and alone[3] is None
    for x, y in zip(out, again):
        assert (x is None and y is None) or torch.equal(x, y)
    assert torch.equal(a, out[0]) and torch.equal(b, out[1]) and torch.equal(alone[0], out[0])


def test_no_rows():
    from paper_2607_28848_amd import rope
    w = torch.ones(64, device="cuda")
    freq = rope.frequencies(64, device="cuda")
    none = torch.empty((0, 2, 64), device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    Q, K = rope.fwd(none, none, pos, freq, q_weight=w, k_weight=w)
    assert Q.shape == K.shape == (0, 2, 64)
    # gradients of no rows of a batch: sums of nothing
    x = torch.randn((3, 2, 64), device="cuda")
    out = rope.bwd(none, none, torch.zeros(3, dtype=torch.int32, device="cuda"), freq, rows=pos, Q=x, K=x, q_weight=w, k_weight=w)
    torch.cuda.synchronize()
    assert bool((out[2] == 0).all()) and bool((out[3] == 0).all())


@pytest.mark.parametrize("nxt", [False, True])
def test_far_positions(nxt):
    """The last position, negative ones and the sign's turn: angles of 2 10^9 radians are as exact as small ones.  The
    64-bit product of position and frequency is off by 2^-53 of up to 2^31, here and in the oracle: 2.4 10^-7."""
    from paper_2607_28848_amd import rope
    pos = torch.tensor([0, 1, -1, 7, (1 << 31) - 1, -(1 << 31), 123456789, 1 << 24, (1 << 24) + 1], dtype=torch.int32).cuda()
    freq = rope.frequencies(128, device="cuda")
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((len(pos), 3, 128), generator=gen).cuda()
    Q, _ = rope.fwd(x, None, pos, freq, interleaved=nxt)
    value, bound = forward(x, pos, freq, None, EPS, nxt, F32)
    far = 2 * 2.0 ** -53 * pos.cpu().double().abs()[:, None, None] * 2 * x.cpu().double().abs().amax()
    check(Q, (value, bound + far), "Q")
    # frequencies of a quarter turn: cosines and sines of 0 and 1 to the bit, at every quarter
    quarter = torch.full((32,), math.pi / 2, dtype=torch.float64, device="cuda")
    y, _ = rope.fwd(torch.ones((8, 1, 64), device="cuda"), None, torch.arange(-4, 4, dtype=torch.int32, device="cuda"), quarter)
    want = torch.tensor([(1, 1), (-1, 1), (-1, -1), (1, -1)] * 2).float()
    assert torch.equal(y.cpu()[:, 0, ::32], want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place(dtype):
    from paper_2607_28848_amd import rope
    gen = torch.Generator().manual_seed(5)
    q, k, v = columns(77, 6, 2, 128, dtype, "fused", gen)
    pos, freq, qw, kw = setting(77, 128, 64, True, gen)
    how = dict(q_weight=qw, k_weight=kw, eps=EPS)
    Q, K = rope.fwd(q, k, pos, freq, **how)
    back = rope.bwd(Q, K, pos, freq, Q=q, K=k, **how)
    dq, dk = Q.clone(), K.clone()
    rope.bwd(dq, dk, pos, freq, Q=q, K=k, dQ_out=dq, dK_out=dk, **how)
    kept = v.clone()
    rope.fwd(q, k, pos, freq, Q_out=q, K_out=k, **how)
    torch.cuda.synchronize()
    assert torch.equal(q, Q) and torch.equal(k, K) and torch.equal(v, kept)
    assert torch.equal(dq, back[0]) and torch.equal(dk, back[1])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinities_stay_where_they_are(dtype):
    """Without a norm an infinite or NaN element reaches its own pair alone, and an unturned one itself alone."""
    from paper_2607_28848_amd import rope
    x = torch.ones((4, 2, 64), dtype=dtype, device="cuda")
    x[1, 0, 40] = math.inf   # unturned
    x[2, 1, 3] = math.nan    # pair (3, 19)
    pos = torch.arange(4, dtype=torch.int32, device="cuda") + 1
    y, _ = rope.fwd(x, None, pos, rope.frequencies(32, device="cuda"))
    bad = ~y.isfinite().cpu()
    want = torch.zeros((4, 2, 64), dtype=torch.bool)
    want[1, 0, 40] = want[2, 1, 3] = want[2, 1, 19] = True
    assert torch.equal(bad, want) and float(y[1, 0, 40]) == math.inf
    g = rope.bwd(x, None, pos, rope.frequencies(32, device="cuda"))[0]
    assert torch.equal(~g.isfinite().cpu(), want)
    # zeros have a norm: eps keeps it finite
    w = torch.ones(64, device="cuda")
    z, _ = rope.fwd(torch.zeros_like(x), None, pos, None, q_weight=w)
    assert bool((z == 0).all())


def test_offsets_past_32_bits():
    """Slots of a cache whose rows lie 4 GiB and more behind its start, in elements and in bytes."""
    from paper_2607_28848_amd import rope
    n_slots, hkv, d = (1 << 31) // 128 // 2 + 64, 2, 128  # a head's rows: 2^30 elements and more; both: past 2^31
    cache = torch.empty((hkv, n_slots, d), dtype=BF, device="cuda")
    K = cache.transpose(0, 1)
    gen = torch.Generator().manual_seed(6)
    k = torch.randn((3, hkv, d), generator=gen).to(BF).cuda()
    slots = torch.tensor([0, n_slots - 1, n_slots // 2], dtype=torch.int32, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    freq = rope.frequencies(d, device="cuda")
    _, want = rope.fwd(None, k, pos, freq)
    rope.fwd(None, k, pos, freq, slots=slots, K_out=K)
    torch.cuda.synchronize()
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(K[s], want[i])


def test_streams_and_graph_replays():
    """Another stream, and a captured forward and backward replayed on new inputs, eager work in between."""
    from paper_2607_28848_amd import rope
    n, hq, hkv, d = 300, 8, 2, 128
    gen = torch.Generator().manual_seed(8)
    q, k, v = columns(n, hq, hkv, d, BF, "fused", gen)
    pos, freq, qw, kw = setting(n, d, d, True, gen)
    rows = torch.arange(0, n, 3, dtype=torch.int32, device="cuda")
    dQ, dK, _ = columns(len(rows), hq, hkv, d, BF, "fused", gen)
    how = dict(q_weight=qw, k_weight=kw, eps=EPS)

    def eager(stream=None):
        return rope.fwd(q, k, pos, freq, V=v, stream=stream, **how) + rope.bwd(dQ, dK, pos, freq, rows=rows, Q=q, K=k, stream=stream,
                                                                             **how)
    first = eager()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for out in (eager(side),):
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, out))
    buf = [t.clone() for t in first]
    ws = torch.empty(rope.workspace_bytes(len(rows), hq, hkv, d), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rope.fwd(q, k, pos, freq, V=v, Q_out=buf[0], K_out=buf[1], V_out=buf[2], **how)
        rope.bwd(dQ, dK, pos, freq, rows=rows, Q=q, K=k, dQ_out=buf[3], dK_out=buf[4], dq_weight=buf[5], dk_weight=buf[6],
                 workspace=ws, **how)
    for seed in range(3):
        for t, b in zip((q, k, v), columns(n, hq, hkv, d, BF, "fused", torch.Generator().manual_seed(30 + seed))):
            t.copy_(b)
        pos.copy_((pos + 1000 * seed) % 4096)
        graph.replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(buf, want))


def test_gradient_against_differences():
    """fp32: the directional derivatives of sum(y dy) by central differences.  A step of 2^-7 along a unit-variance
    direction leaves an error of third order, below 8 h^2 of the terms' absolute sum."""
    from paper_2607_28848_amd import rope
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((20, 3, 64), generator=gen, device="cuda")
    w = 1 + 0.2 * torch.randn((64,), generator=gen, device="cuda")
    dy = torch.randn((20, 3, 64), generator=gen, device="cuda")
    pos = torch.arange(20, dtype=torch.int32, device="cuda") * 37
    freq = rope.frequencies(32, device="cuda")

    def L(x, w):
        return float((rope.fwd(x, None, pos, freq, q_weight=w, interleaved=True)[0].double() * dy.double()).sum())

    dx, _, dw, _ = rope.bwd(dy, None, pos, freq, Q=x, q_weight=w, interleaved=True)
    h = 2.0 ** -7
    for i, grad in ((0, dx), (1, dw)):
        u = torch.randn((x, w)[i].shape, generator=gen, device="cuda")
        a, b = [x, w], [x, w]
        a[i], b[i] = a[i] + h * u, b[i] - h * u
        num = (L(*a) - L(*b)) / (2 * h)
        ana = float((grad.double() * u.double()).sum())
        size = float((grad.double() * u.double()).abs().sum()) + float((dy.double() * w.double()).abs().sum()) * 2.0 ** -4
        assert abs(num - ana) <= 8 * h * h * size + 1e-4, (i, num, ana, size)
