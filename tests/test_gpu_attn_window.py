"""Attention with a window and sinks on the GPU against the 64-bit oracle: windows and sinks around the tiles' edges, from
one token to thousands, queries that see nothing, garbage in rows that no query sees, gradients, graphs and long caches."""
import math

import pytest
import torch

from attn_util import check
from test_gpu_attn import MIXED, place, tensors
from window_util import oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def unseen(seqs, window, sinks, n_kv):
    """Rows of K and V that some sequence holds but no query of any sees."""
    held, seen = torch.zeros(n_kv, dtype=torch.bool), torch.zeros(n_kv, dtype=torch.bool)
    for _, ql, k0, kl, _ in seqs:
        held[k0:k0 + kl] = True
        if ql == 0:
            continue
        seen[k0:k0 + min(kl, sinks)] = True
        seen[k0 + max(0, min(kl, kl - ql + 1 - window)):k0 + kl] = True
    return held & ~seen


def run(seqs, nq, nk, hq, hkv, d, dtype, layout, window, sinks, seed=0, garbage=math.nan, q_std=2.0):
    from paper_2607_28848_amd import attn
    scale = 1 / math.sqrt(d)
    Q, K, V = tensors(seqs, nq, nk, hq, hkv, d, dtype, layout, seed, q_std)
    hidden = unseen(seqs, window, sinks, nk).cuda()
    clean = [t.clone() for t in (K, V)]
    if layout != "fused":  # a fused row's hidden keys are beside queries
        K[hidden], V[hidden] = garbage, garbage
        for t in clean:
            t[hidden] = 0.0
    plan = attn.Plan(seqs, nq, nk, hq, hkv, d, device="cuda", window=window, sinks=sinks)
    mark = 7.0  # what no sequence's rows hold must stay
    O = torch.full((nq, hq, d), mark, dtype=dtype, device="cuda")
    lse = torch.full((hq, nq), mark, device="cuda")
    attn.fwd(plan, Q, K, V, scale=scale, O=O, lse=lse)
    held = torch.zeros(nq, dtype=torch.bool)
    for q0, ql, *_ in seqs:
        held[q0:q0 + ql] = True
    assert bool((O.cpu()[~held] == mark).all()) and bool((lse.cpu()[:, ~held] == mark).all())
    dO = torch.randn((plan.train_q, hq, d), generator=torch.Generator().manual_seed(seed + 1)).to(dtype).cuda()
    want = oracle(seqs, Q, *clean, scale, window, sinks, dO)
    got = {"O": O, "lse": lse}
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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (31, 0), (64, 64), (65, 4), (100, 33), (128, 130), (250, 1)])
@pytest.mark.parametrize("hq,hkv,d,layout", [(4, 2, 128, "cache"), (3, 3, 64, "heads"), (7, 1, 128, "fused")])
def test_mixed_batch(dtype, window, sinks, hq, hkv, d, layout):
    print(dtype, window, sinks, hq, hkv, d, layout, flush=True)
    run(*place(MIXED, layout, q_gap=2), hq, hkv, d, dtype, layout, window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 2), (37, 0), (64, 4), (129, 16), (700, 70), (1000, 5000)])
@pytest.mark.parametrize("lens", [[(1, 5000, 0)], [(5, 1031, 0), (1, 64, 0), (16, 4097, 0)], [(300, 2500, 0)], [(700, 700, 1)],
                                  [(257, 811, 1), (384, 384, 1)], [(200, 3000, 1)], [(1400, 1400, 1)], [(500, 13, 1)]])
def test_lengths(lens, window, sinks, d):
    print(lens, window, sinks, d, flush=True)
    run(*place(lens, "cache"), 4, 2, d, BF, "cache", window, sinks, seed=3)


@pytest.mark.parametrize("lens", [[(1, 900, 0)], [(300, 700, 1)], [(20, 333, 1)]])
@pytest.mark.parametrize("window,sinks", [(1, 2), (37, 0), (64, 4), (129, 17)])
def test_lengths_f32(lens, window, sinks):
    run(*place(lens, "cache"), 4, 2, 128, F32, "cache", window, sinks, seed=3)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_hidden_infinities(dtype):
    """Infinite keys and values that no query sees, and a window that a scaled row's largest score lies outside of."""
    run(*place([(150, 450, 1), (1, 400, 0), (10, 333, 0)], "cache"), 4, 2, 64, dtype, "cache", 70, 5, garbage=math.inf, q_std=20.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_order_of_the_table_and_shared_keys(dtype):
    seqs = [(150, 60, 0, 100, 1), (10, 80, 40, 80, 1), (100, 1, 0, 120, 0), (0, 10, 0, 90, 1)]
    run(seqs, 220, 130, 4, 2, 128, dtype, "cache", 33, 6, seed=5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_wide_windows_give_the_plain_results(dtype):
    """A window that hides nothing: the same bits as without one; one that hides a single key of one sequence: the other
    sequences' results are within the bounds, that one's differ."""
    from paper_2607_28848_amd import attn
    seqs, nq, nk = place([(150, 300, 1), (1, 500, 0), (64, 64, 1)], "cache")
    Q, K, V = tensors(seqs, nq, nk, 4, 2, 64, dtype, "cache")
    dO = torch.randn((214, 4, 64), device="cuda").to(dtype)
    outs = []
    for w, s in ((None, 0), (500, 0), (3, 497), ((1 << 31) - 1, (1 << 31) - 1), (499, 0)):
        plan = attn.Plan(seqs, nq, nk, 4, 2, 64, device="cuda", window=w, sinks=s)
        O, lse = attn.fwd(plan, Q, K, V)
        outs.append((O, lse, *attn.bwd(plan, Q, K, V, O, lse, dO)))
    torch.cuda.synchronize()
    for other in outs[1:4]:
        assert all(torch.equal(x, y) for x, y in zip(outs[0], other))
    one = seqs[1][0]
    assert not torch.equal(outs[0][1][:, one], outs[4][1][:, one])
    run(seqs, nq, nk, 4, 2, 64, dtype, "cache", 499, 0)


def test_pieces_of_long_samples():
    """Few heads, so that query tiles and the sinks' key tile are cut into pieces."""
    run(*place([(2300, 2300, 1)], "cache"), 2, 1, 128, BF, "cache", 300, 4, seed=11)
    run(*place([(3000, 3000, 1)], "fused"), 1, 1, 64, BF, "fused", 1500, 130, seed=12)


def test_a_trimmed_cache():
    """The sinks' and the last window's keys moved together give what the whole cache gives."""
    from paper_2607_28848_amd import attn
    window, sinks, kl, d = 200, 4, 3000, 128
    g = torch.Generator().manual_seed(4)
    Q = torch.randn((1, 8, d), generator=g).to(BF).cuda()
    K, V = (torch.randn((kl, 2, d), generator=g).to(BF).cuda() for _ in range(2))
    kept = torch.cat((torch.arange(sinks), torch.arange(kl - window, kl))).cuda()
    O, lse = attn.fwd(attn.Plan([(0, 1, 0, kl, 0)], 1, kl, 8, 2, d, device="cuda", window=window, sinks=sinks), Q, K, V)
    n = len(kept)
    O2, lse2 = attn.fwd(attn.Plan([(0, 1, 0, n, 0)], 1, n, 8, 2, d, device="cuda", window=window, sinks=sinks), Q, K[kept].contiguous(),
                        V[kept].contiguous())
    want = oracle([(0, 1, 0, kl, 0)], Q, K, V, 1 / math.sqrt(d), window, sinks)
    torch.cuda.synchronize()
    for o, l in ((O, lse), (O2, lse2)):
        check(o, want["O"], "O")
        check(l, want["lse"], "lse")


def test_repeats_streams_and_replays():
    """The same bits from call to call and on another stream; a captured step replayed on new inputs, two graphs on one
    workspace, eager work in between."""
    from paper_2607_28848_amd import attn
    seqs, nq, nk = place([(1, 3000, 0), (200, 200, 1), (40, 900, 1)], "cache")
    plan = attn.Plan(seqs, nq, nk, 8, 2, 128, device="cuda", window=150, sinks=4)
    ws = torch.empty(attn.workspace_bytes(plan, BF), dtype=torch.uint8, device="cuda")
    Q, K, V = (t.clone() for t in tensors(seqs, nq, nk, 8, 2, 128, BF, "cache"))
    dO = torch.randn((plan.train_q, 8, 128), device="cuda").to(BF)

    def eager(stream=None):
        O, lse = attn.fwd(plan, Q, K, V, stream=stream)
        return (O, lse) + attn.bwd(plan, Q, K, V, O, lse, dO, stream=stream)

    first = eager()
    torch.cuda.synchronize()
    again, other = eager(), eager(torch.cuda.Stream())
    torch.cuda.synchronize()
    for x, y, z in zip(first, again, other):
        assert torch.equal(x, y) and torch.equal(x, z)
    bufs, graphs = [], []
    for _ in range(2):
        b = [t.clone() for t in first]
        bufs.append(b)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attn.fwd(plan, Q, K, V, O=b[0], lse=b[1], workspace=ws)
            attn.bwd(plan, Q, K, V, b[0], b[1], dO, dQ=b[2], dK=b[3], dV=b[4], workspace=ws)
        graphs.append(g)
    for seed in range(3):
        for t, n in zip((Q, K, V), tensors(seqs, nq, nk, 8, 2, 128, BF, "cache", seed=seed + 20)):
            t.copy_(n)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        for b in bufs:
            for x, y in zip(b, want):
                assert bool(((x == y) | (x.isnan() & y.isnan())).all())


def test_offsets_past_32_bits():
    """The window of a long cache that lies past 2^31 elements of its head."""
    from paper_2607_28848_amd import attn
    kl, d, window, sinks = (1 << 31) // 128 + 5000, 128, 300, 4
    K, V = (torch.zeros((kl, 1, d), dtype=BF, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(6)
    for t in (K, V):
        t[-600:] = torch.randn((600, 1, d), generator=g).to(BF)
        t[:10] = torch.randn((10, 1, d), generator=g).to(BF)
    Q = torch.randn((41, 4, d), generator=g).to(BF).cuda()
    small = torch.cat((torch.arange(10), torch.arange(kl - 600, kl))).cuda()
    k, v = K[small], V[small]
    for ql in (1, 41):
        O, lse = attn.fwd(attn.Plan([(0, ql, 0, kl, 0)], 41, kl, 4, 1, d, device="cuda", window=window, sinks=sinks), Q, K, V)
        want = oracle([(0, ql, 0, 610, 0)], Q, k, v, 1 / math.sqrt(d), window, sinks)
        torch.cuda.synchronize()
        check(O[:ql], tuple(t[:ql] for t in want["O"]), "O")
        check(lse[:, :ql], tuple(t[:, :ql] for t in want["lse"]), "lse")


def test_gradient_against_differences():
    """fp32: the directional derivatives of sum(O dO) by central differences, as for attention without a window."""
    from paper_2607_28848_amd import attn
    seqs, nq, nk = place([(40, 40, 1), (21, 70, 1)], "cache")
    Q, K, V = (t.nan_to_num(nan=0.0) for t in tensors(seqs, nq, nk, 4, 2, 64, F32, "cache", q_std=1.0))
    plan = attn.Plan(seqs, nq, nk, 4, 2, 64, device="cuda", window=9, sinks=2)
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
