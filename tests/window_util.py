"""The oracle of attention with a window and sinks: softmax attention and its gradients in 64 bits on the CPU, head by
head, with the bounds of attn_util (their terms hold for any set of keys that a row sees)."""
import math

import torch

from attn_util import E32, EXTRA, unit


def oracle(seqs, Q, K, V, scale, window, sinks, dO=None):
    """dict of (value, bound) for O, lse and, given dO (compact rows), dQ, dK, dV."""
    u = unit(Q.dtype)
    Q, K, V = (t.detach().cpu().double() for t in (Q, K, V))
    hq, d, hkv = Q.shape[1], Q.shape[2], K.shape[1]
    group = hq // hkv
    O, Ob = torch.zeros_like(Q), torch.zeros_like(Q)
    lse, lseb = torch.full((hq, Q.shape[0]), -math.inf, dtype=torch.float64), torch.zeros((hq, Q.shape[0]), dtype=torch.float64)
    train = sorted((s for s in seqs if s[4]), key=lambda s: s[0])
    nq, nk = sum(s[1] for s in train), sum(s[3] for s in train)
    if dO is not None:
        dO = dO.detach().cpu().double()
        dQ, dQb = (torch.zeros((nq, hq, d), dtype=torch.float64) for _ in range(2))
        dK, dKb, dV, dVb = (torch.zeros((nk, hkv, d), dtype=torch.float64) for _ in range(4))
    cq = ck = 0
    for q0, ql, k0, kl, tr in sorted(seqs, key=lambda s: s[0]):
        for h in range(hq if ql and kl else 0):
            g = h // group
            q, k, v = Q[q0:q0 + ql, h], K[k0:k0 + kl, g], V[k0:k0 + kl, g]
            j, p_ = torch.arange(kl)[None, :], torch.arange(ql)[:, None] + (kl - ql)
            see = (j <= p_) & ((j > p_ - window) | (j < sinks))
            some = see.any(dim=1)
            s = torch.where(see, q @ k.t() * scale, -math.inf)
            es = torch.where(see, ((d + 4) * scale * (q.abs() @ k.abs().t()) + 4 * s.abs()) * E32, 0.0)
            esm = es.amax(dim=1)
            n = torch.logsumexp(s, dim=1)
            p = torch.where(see, torch.exp(s - torch.where(some, n, 0.0)[:, None]), 0.0)
            r = es + (esm + (kl + 16) * E32 + u)[:, None]
            o = p @ v
            O[q0:q0 + ql, h] = o
            Ob[q0:q0 + ql, h] = EXTRA * ((p * r) @ v.abs() + u * o.abs()) + 1e-30
            lse[h, q0:q0 + ql] = n
            lseb[h, q0:q0 + ql] = EXTRA * (esm + (kl + 16) * E32 + 4 * E32 * torch.where(some, n.abs(), 0.0))
            if dO is None or not tr:
                continue
            w = dO[cq:cq + ql, h]
            dp = w @ v.t()
            delta = (w * o).sum(dim=1)
            ds = p * (dp - delta[:, None]) * scale
            # delta is formed from the rounded output; dp and delta are fp32 sums
            eps_delta = (w.abs() * Ob[q0:q0 + ql, h]).sum(dim=1) + d * E32 * (w.abs() * o.abs()).sum(dim=1)
            eps_dp = d * E32 * (w.abs() @ v.abs().t())
            eds = ds.abs() * (r + 4 * u) + p * scale * (eps_dp + eps_delta[:, None]) * (1 + r)
            dQ[cq:cq + ql, h] = ds @ k
            dQb[cq:cq + ql, h] = EXTRA * ((eds + kl * E32 * ds.abs()) @ k.abs() + u * (ds @ k).abs()) + 1e-30
            dK[ck:ck + kl, g] += ds.t() @ q
            dKb[ck:ck + kl, g] += EXTRA * (eds + group * ql * E32 * ds.abs()).t() @ q.abs() + 1e-30
            dV[ck:ck + kl, g] += p.t() @ w
            dVb[ck:ck + kl, g] += EXTRA * (p * (r + group * ql * E32)).t() @ w.abs() + 1e-30
        if tr:
            cq, ck = cq + ql, ck + kl
    out = {"O": (O, Ob), "lse": (lse, lseb)}
    if dO is not None:
        out.update(dQ=(dQ, dQb), dK=(dK, dKb + EXTRA * u * dK.abs()), dV=(dV, dVb + EXTRA * u * dV.abs()))
    return out
