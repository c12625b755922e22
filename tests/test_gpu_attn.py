"""Attention of a mixed batch on the GPU against the 64-bit oracle: lengths from none to thousands, head layouts,
storage layouts, rows that see nothing, garbage around what may be read, gradients, and repeatability."""
import math

import pytest
import torch

from attn_util import check, oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def place(lens, layout, q_gap=0):
    """[(q_len, k_len, train)] -> (sequences, n_q, n_kv); "fused": K and V rows are the rows of Q."""
    seqs, nq, nk = [], q_gap, 3
    for ql, kl, tr in lens:
        seqs.append((nq, ql, nq if layout == "fused" else nk, kl, tr))
        nq += max(ql, kl if layout == "fused" else 0) + q_gap
        nk += kl + 5
    return seqs, nq + 1, nq + 1 if layout == "fused" else nk + 2


def tensors(seqs, nq, nk, hq, hkv, d, dtype, layout, seed=0, q_std=2.0):
    """Q, K, V as a caller has them; every row that no sequence holds is NaN."""
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.full(s, math.nan) for s in ((nq, hq, d), (nk, hkv, d), (nk, hkv, d)))
    for q0, ql, k0, kl, _ in seqs:
        q[q0:q0 + ql] = torch.randn((ql, hq, d), generator=g) * q_std
        k[k0:k0 + kl] = torch.randn((kl, hkv, d), generator=g)
        v[k0:k0 + kl] = torch.randn((kl, hkv, d), generator=g)
    q, k, v = (t.to(dtype).cuda() for t in (q, k, v))
    if layout == "fused":
        rows = torch.cat((q, k, v), dim=1)
        return rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    if layout == "heads":
        return q.transpose(0, 1).contiguous().transpose(0, 1), *(t.transpose(0, 1).contiguous().transpose(0, 1) for t in (k, v))
    if layout == "padded":  # rows and heads further apart than they are long
        def pad(t):
            b = torch.full((t.shape[0], t.shape[1] + 1, d + 8), math.nan, dtype=dtype, device="cuda")
            b[:, :t.shape[1], :d] = t
            return b[:, :t.shape[1], :d]
        return pad(q), pad(k), pad(v)
    return q, k, v


def run(seqs, nq, nk, hq, hkv, d, dtype, layout, seed=0, scale=None, grads=True, q_std=2.0):
    from paper_2607_28848_amd import attn
    scale = 1 / math.sqrt(d) if scale is None else scale
    Q, K, V = tensors(seqs, nq, nk, hq, hkv, d, dtype, layout, seed, q_std)
    plan = attn.Plan(seqs, nq, nk, hq, hkv, d, device="cuda")
    mark = 7.0  # what no sequence's rows hold must stay
    O = torch.full((nq, hq, d), mark, dtype=dtype, device="cuda")
    lse = torch.full((hq, nq), mark, device="cuda")
    attn.fwd(plan, Q, K, V, scale=scale, O=O, lse=lse)
    held = torch.zeros(nq, dtype=torch.bool)
    for q0, ql, *_ in seqs:
        held[q0:q0 + ql] = True
    assert bool((O.cpu()[~held] == mark).all()) and bool((lse.cpu()[:, ~held] == mark).all())
    dO = torch.randn((plan.train_q, hq, d), generator=torch.Generator().manual_seed(seed + 1)).to(dtype).cuda()
    want = oracle(seqs, Q, K, V, scale, dO if grads else None)
    got = {"O": O, "lse": lse}
    if grads:
        got.update(zip(("dQ", "dK", "dV"), attn.bwd(plan, Q, K, V, O, lse, dO, scale=scale)))
    torch.cuda.synchronize()
    for name, t in got.items():
        value, bound = want[name]
        if name == "O":
            t, value, bound = t[held], value[held], bound[held]
        elif name == "lse":
            t, value, bound = t[:, held], value[:, held], bound[:, held]
        check(t, (value, bound), name)
    return got


# query lengths around the tiles and the split form's limit, keys behind, level with and short of them, none at all
MIXED = [(1, 1, 0), (33, 33, 1), (0, 9, 0), (1, 77, 0), (16, 40, 1), (17, 17, 0), (130, 130, 1), (9, 0, 0), (65, 200, 1),
         (20, 7, 1), (3, 2, 0), (128, 129, 0), (0, 0, 1), (70, 0, 1), (1, 300, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,d,layout", [(4, 2, 128, "cache"), (3, 3, 64, "heads"), (7, 1, 128, "fused"),
                                             (8, 2, 64, "padded"), (40, 1, 64, "cache"), (1, 1, 128, "heads")])
def test_mixed_batch(dtype, hq, hkv, d, layout):
    print(dtype, hq, hkv, d, layout, flush=True)
    run(*place(MIXED, layout, q_gap=2), hq, hkv, d, dtype, layout)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(1, 1, 1)], [(1, 5000, 0)], [(5, 1031, 0), (1, 64, 0), (16, 4097, 0)],
                                  [(1, 127, 0)] * 3 + [(1, 129, 0)] * 3, [(300, 2500, 0)], [(700, 700, 1)],
                                  [(257, 511, 1), (384, 384, 1)], [(2, 1, 1)], [(500, 13, 1)]])
def test_lengths(lens, d):
    print(lens, d, flush=True)
    run(*place(lens, "cache"), 4, 2, d, BF, "cache", seed=3)


def test_order_of_the_table_and_shared_keys():
    """Sequences out of order in the table; three of them on one prefix's key rows."""
    seqs = [(150, 60, 0, 100, 1), (10, 80, 40, 80, 1), (100, 1, 0, 120, 0), (0, 10, 0, 90, 1)]
    for dtype in (BF, F32):
        run(seqs, 220, 130, 4, 2, 128, dtype, "cache", seed=5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale,q_std", [(1.0, 4.0), (1e-3, 1.0), (0.25, 30.0)])
def test_scales(dtype, scale, q_std):
    """Flat rows, and scores of hundreds, whose reference moves from block to block."""
    run(*place([(150, 350, 1), (1, 400, 0), (64, 64, 1)], "cache"), 4, 4, 64, dtype, "cache", seed=9, scale=scale, q_std=q_std)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rising_scores(dtype):
    """Keys whose scores rise along the row, so that the running maximum moves at every block, and a query of zeros."""
    from paper_2607_28848_amd import attn
    n, d = 700, 64
    Q = torch.zeros((n, 1, d))
    Q[:, 0, 0] = torch.arange(n) % 3
    K = torch.zeros((n, 1, d))
    K[:, 0, 0] = torch.arange(n) / 4
    V = torch.randn((n, 1, d), generator=torch.Generator().manual_seed(2))
    Q, K, V = (t.to(dtype).cuda() for t in (Q, K, V))
    seqs = [(0, n - 1, 0, n - 1, 0), (n - 1, 1, 0, n, 0)]
    O, lse = attn.fwd(attn.Plan(seqs, n, n, 1, 1, d, device="cuda"), Q, K, V, scale=1.0)
    want = oracle(seqs, Q, K, V, 1.0)
    check(O, want["O"], "O")
    check(lse, want["lse"], "lse")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_scores_and_masked_keys(dtype):
    """Keys of -infinity scores drop out; what a masked key holds reaches no score of the rows that do not see it."""
    from paper_2607_28848_amd import attn
    n, d = 200, 64
    g = torch.Generator().manual_seed(4)
    Q, K, V = (torch.randn((n, 2, d), generator=g).to(dtype) for _ in range(3))
    Q[:, :, 0] = 1.0
    K[50:60, :, 0] = -math.inf
    K[150, :, 1] = math.nan  # the rows from 150 on see it
    seqs = [(0, n, 0, n, 0)]
    O, lse = attn.fwd(attn.Plan(seqs, n, n, 2, 2, d, device="cuda"), Q.cuda(), K.cuda(), V.cuda())
    k = K.clone()
    k[150, :, 1] = 0
    want = {name: (v.clone(), b) for name, (v, b) in oracle(seqs, Q, torch.where(k.isinf(), -1e4, k.float()).to(dtype), V,
                                                            1 / math.sqrt(d)).items()}
    b = want["O"][1].nan_to_num(nan=0.0)
    assert bool((O[150:].isnan()).all()) and bool(lse[:, 150:].isnan().all())
    # the stand-in's huge score widens the oracle's bound: plain rounding of p and o is what is left
    u = 2.0 ** -8 if dtype == BF else 2.0 ** -18
    bound = u * (want["O"][0].abs() + V.abs().max().double())
    check(O[:150], (want["O"][0][:150], bound[:150]), "O")
    assert b.shape == O.shape


@pytest.mark.parametrize("dtype", [BF, F32])
def test_repeats_and_streams(dtype):
    """The same bits from call to call, on another stream, and with other work beside it."""
    from paper_2607_28848_amd import attn
    seqs, nq, nk = place([(1, 3000, 0), (200, 200, 1), (40, 900, 1)], "cache")
    Q, K, V = tensors(seqs, nq, nk, 8, 2, 128, dtype, "cache")
    plan = attn.Plan(seqs, nq, nk, 8, 2, 128, device="cuda")
    dO = torch.randn((plan.train_q, 8, 128), device="cuda").to(dtype)
    O, lse = attn.fwd(plan, Q, K, V)
    first = (O, lse) + attn.bwd(plan, Q, K, V, O, lse, dO)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (None, side):
        with torch.cuda.stream(s or torch.cuda.current_stream()):
            O, lse = attn.fwd(plan, Q, K, V)
            again = (O, lse) + attn.bwd(plan, Q, K, V, O, lse, dO)
        torch.cuda.synchronize()
        for x, y in zip(first, again):
            assert bool(((x == y) | (x.isnan() & y.isnan())).all())


def test_graph_replays():
    """Forward and backward captured once and replayed on new inputs, eager work in between."""
    from paper_2607_28848_amd import attn
    seqs, nq, nk = place([(1, 900, 0), (130, 130, 1), (60, 300, 0)], "cache")
    plan = attn.Plan(seqs, nq, nk, 4, 2, 64, device="cuda")
    ws = torch.empty(attn.workspace_bytes(plan, BF), dtype=torch.uint8, device="cuda")
    base = tensors(seqs, nq, nk, 4, 2, 64, BF, "cache")
    Q, K, V = (t.clone() for t in base)
    dO = torch.randn((plan.train_q, 4, 64), device="cuda").to(BF)
    O, lse = attn.fwd(plan, Q, K, V, workspace=ws)
    g = attn.bwd(plan, Q, K, V, O, lse, dO, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.fwd(plan, Q, K, V, O=O, lse=lse, workspace=ws)
        attn.bwd(plan, Q, K, V, O, lse, dO, dQ=g[0], dK=g[1], dV=g[2], workspace=ws)
    for seed in range(3):
        for t, b in zip((Q, K, V), tensors(seqs, nq, nk, 4, 2, 64, BF, "cache", seed=seed + 20)):
            t.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        eO, else_ = attn.fwd(plan, Q, K, V)
        eg = attn.bwd(plan, Q, K, V, eO, else_, dO)
        torch.cuda.synchronize()
        for q0, ql, *_ in seqs:
            assert torch.equal(O[q0:q0 + ql], eO[q0:q0 + ql]) and torch.equal(lse[:, q0:q0 + ql], else_[:, q0:q0 + ql])
        for x, y in zip(g, eg):
            assert torch.equal(x, y)


def test_gradient_against_differences():
    """fp32: the directional derivatives of sum(O dO) by central differences.  A step of 2^-6 along a unit-variance
    direction leaves an error of third order (about h^2 times the derivative) and 2^-24 |L| / h of rounding."""
    from paper_2607_28848_amd import attn
    seqs, nq, nk = place([(40, 40, 1), (21, 70, 1)], "cache")
    Q, K, V = (t.nan_to_num(nan=0.0) for t in tensors(seqs, nq, nk, 4, 2, 64, F32, "cache", q_std=1.0))
    plan = attn.Plan(seqs, nq, nk, 4, 2, 64, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(8)
    dO = torch.randn((plan.train_q, 4, 64), generator=gen, device="cuda")
    rows = [i for q0, ql, *_ in seqs for i in range(q0, q0 + ql)]
    keys = [i for _, _, k0, kl, _ in seqs for i in range(k0, k0 + kl)]

    def L(q, k, v):
        return float((attn.fwd(plan, q, k, v)[0][rows].double() * dO.double()).sum())

    O, lse = attn.fwd(plan, Q, K, V)
    grads = attn.bwd(plan, Q, K, V, O, lse, dO)
    h = 2.0 ** -6
    for i, (grad, idx) in enumerate(zip(grads, (rows, keys, keys))):
        u = torch.randn((Q, K, V)[i].shape, generator=gen, device="cuda")
        a, b = [Q, K, V], [Q, K, V]
        a[i], b[i] = a[i] + h * u, b[i] - h * u
        num = (L(*a) - L(*b)) / (2 * h)
        ana = float((grad.double() * u[idx].double()).sum())
        size = float((grad.double() * u[idx].double()).abs().sum())
        assert abs(num - ana) <= 8 * h * h * size, (i, num, ana, size)
