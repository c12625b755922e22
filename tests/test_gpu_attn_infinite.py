"""Gradients where scores are -infinity: such a key has no part in any sum.  The keys in front of each sequence hold
-infinity in one element, which every query meets with a positive one; without them the sequence is an ordinary one, and
that is what the outputs are held against.  (dQ has 0 times that -infinity, NaN, in that element, which is left out.)"""
import math

import pytest
import torch

from attn_util import check, oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql,kl,gone", [(40, 46, 6), (64, 65, 1), (150, 250, 70), (131, 140, 3), (9, 13, 4), (1, 2, 1)])
def test_keys_of_minus_infinity(dtype, d, ql, kl, gone):
    run(dtype, d, ql, kl, gone)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql,kl,gone", [(40, 40, 6), (64, 64, 1), (150, 150, 70), (131, 131, 131), (9, 9, 4), (1, 1, 1),
                                        (200, 140, 20), (700, 700, 300)])
def test_queries_of_no_other_keys(dtype, d, ql, kl, gone):
    """The first queries see only such keys, and count as if they saw none."""
    run(dtype, d, ql, kl, gone)


def run(dtype, d, ql, kl, gone):
    from paper_2607_28848_amd import attn
    hq, hkv = 4, 2
    g = torch.Generator().manual_seed(kl + d)
    q, k, v, do = (torch.randn((n, h, d), generator=g).to(dtype) for n, h in ((ql, hq), (kl, hkv), (kl, hkv), (ql, hq)))
    q[:, :, 0] = 0.5 + q[:, :, 0].abs()
    k[:gone, :, 0] = -math.inf
    q, k, v, do = (t.cuda() for t in (q, k, v, do))
    plan = attn.Plan([(0, ql, 0, kl, 1)], ql, kl, hq, hkv, d, device="cuda")
    o, lse = attn.fwd(plan, q, k, v)
    dq, dk, dv = attn.bwd(plan, q, k, v, o, lse, do)
    k0 = k.clone()
    k0[:gone] = 0
    want = oracle([(0, ql, gone, kl - gone, 1)], q, k0, v, 1 / math.sqrt(d), do)
    check(o, want["O"], "O")
    check(lse, want["lse"], "lse")
    alone = (lse == -math.inf).all(dim=0)
    assert bool((alone.cpu() == (torch.arange(ql) < gone + ql - kl)).all())
    assert bool((dq[alone] == 0).all())
    check(dq[~alone][:, :, 1:], tuple(t[~alone.cpu()][:, :, 1:] for t in want["dQ"]), "dQ")
    for name, t in (("dK", dk), ("dV", dv)):
        check(t[gone:], want[name], name)
        assert bool((t[:gone] == 0).all()), name
