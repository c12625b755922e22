"""Attention calls at the limits of their arguments: what is refused, and addresses that 32 bits do not hold."""
import math

import pytest
import torch

from attn_util import check, oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def test_refusals():
    from paper_2607_28848_amd import attn, dsv
    lib = dsv.lib_handle()
    seqs, nq, nk, hq, hkv, d = [(0, 40, 0, 40, 1), (40, 1, 40, 500, 0)], 41, 540, 4, 2, 64
    plan = attn.Plan(seqs, nq, nk, hq, hkv, d, device="cuda")
    room = 64  # rows to spare, for the strides below that are larger than the tensors need
    t = {n: torch.zeros((rows + room, h, d), dtype=BF, device="cuda") for n, rows, h in (
        ("Q", nq, hq), ("K", nk, hkv), ("V", nk, hkv), ("O", nq, hq), ("dO", 40, hq), ("dQ", 40, hq), ("dK", 40, hkv),
        ("dV", 40, hkv))}
    lse = torch.zeros((hq, nq), device="cuda")
    ws = torch.empty(attn.workspace_bytes(plan, BF), dtype=torch.uint8, device="cuda")

    def call(back, dt=0, scale=0.125, lse_at=lse.data_ptr(), ws_at=ws.data_ptr(), n=ws.numel(), **views):
        v = {k: attn.View(x.data_ptr(), 0, 0) for k, x in t.items()}
        v.update({k: attn.View(t[k].data_ptr() + off, row, head) for k, (off, row, head) in views.items()})
        v = list(v.values())
        if back:
            return lib.dsv_attn_bwd(plan.handle, dt, scale, *v[:4], lse_at, *v[4:], ws_at, n, None)
        return lib.dsv_attn_fwd(plan.handle, dt, scale, *v[:4], lse_at, ws_at, n, None)

    arg, size, rng = dsv.ERR_ARG, dsv.ERR_SIZE, dsv.ERR_RANGE
    both = [(dict(dt=2), rng), (dict(scale=math.nan), rng), (dict(scale=math.inf), rng), (dict(scale=0.0), rng),
            (dict(scale=-0.125), rng), (dict(scale=1e300), rng), (dict(lse_at=lse.data_ptr() + 2), arg),
            (dict(ws_at=None), arg), (dict(ws_at=ws.data_ptr() + 16), arg), (dict(n=ws.numel() - 1), size),
            (dict(Q=(2, 0, 0)), arg), (dict(K=(8, 0, 0)), arg), (dict(V=(0, 60, 0)), size), (dict(V=(0, 0, 56)), size),
            (dict(K=(0, 132, 0)), size), (dict(K=(0, 0, 68)), size), (dict(Q=(0, -256, 0)), size),
            (dict(K=(0, (1 << 23) + 8, 0)), size), (dict(K=(0, 0, (1 << 40) + 8)), size)]
    for back in (False, True):
        for kw, want in both:
            assert call(back, **kw) == want, (back, kw)
    # outputs whose vectors overlap
    assert call(False, O=(0, 128, 64)) == size
    for name in ("dQ", "dK", "dV"):
        assert call(True, **{name: (0, 64, 64)}) == size
    assert call(True, lse_at=None) == arg
    assert call(False, lse_at=None) == dsv.OK and call(False) == dsv.OK and call(True) == dsv.OK
    # a row of K that is the same for every key head is an input like any other
    assert call(False, K=(0, 64, 64)) == dsv.OK
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", ["rows", "heads", "row_stride"])
def test_far_addresses(dtype, far):
    """Keys, values and outputs more than 2^31 elements from their tensor's start, on either side of a launch's forms:
    many queries, few queries, a fine-tuning sample."""
    from paper_2607_28848_amd import attn
    hq, hkv, d, lens = 4, 2, 128, [(70, 70, 1), (5, 300, 0), (130, 140, 0)]
    base = (1 << 31) // (hkv * d) if far == "rows" else 0  # first key row that is used
    seqs, q0, k0 = [], 0, base
    for ql, kl, tr in lens:
        seqs.append((q0, ql, k0, kl, tr))
        q0, k0 = q0 + ql, k0 + kl
    nq, nk = q0, k0

    def wide(rows, heads):
        """[rows][heads][d] in far-apart memory; only what `seqs` names is filled."""
        if far == "rows":
            return torch.empty((rows, heads, d), dtype=dtype, device="cuda")
        if far == "heads":
            step = (1 << 31) + 64
            return torch.empty((heads - 1) * step + rows * d, dtype=dtype, device="cuda").as_strided((rows, heads, d),
                                                                                                    (d, step, 1))
        step = 1 << 23
        return torch.empty((rows - 1) * step + heads * d, dtype=dtype, device="cuda").as_strided((rows, heads, d),
                                                                                                (step, d, 1))

    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((n, h, d), generator=g).to(dtype) for n, h in ((nq, hq), (nk - base, hkv), (nk - base, hkv)))
    Q, K, V = q.cuda(), wide(nk, hkv), wide(nk, hkv)
    K[base:], V[base:] = k.cuda(), v.cuda()
    O = wide(nq, hq)
    plan = attn.Plan(seqs, nq, nk, hq, hkv, d, device="cuda")
    _, lse = attn.fwd(plan, Q, K, V, O=O, lse=torch.empty((hq, nq), device="cuda"))
    dO = torch.randn((plan.train_q, hq, d), generator=g).to(dtype).cuda()
    dK, dV = (wide(plan.train_k, hkv) for _ in range(2))
    dQ, dK, dV = attn.bwd(plan, Q, K, V, O, lse, dO, dK=dK, dV=dV)
    near = [(a, b, c - base, e, f) for a, b, c, e, f in seqs]
    want = oracle(near, q, k, v, 1 / math.sqrt(d), dO)
    for name, got in (("O", O), ("lse", lse), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        check(got.contiguous(), want[name], name)
