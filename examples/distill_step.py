#!/usr/bin/env python3
"""One co-batched step of a block with normalised, rotated queries and keys, windowed attention and a teacher.

The step of mixed_step.py with what stands around its attention and loss in many models: queries and keys go through a norm
of each head and the position rotation on their way from the q/k/v product to the attention, which writes keys and values to
the cache's slots; the attention looks back over a window, the first tokens staying visible; and the fine-tuning samples
learn from a teacher's top logits.  The backward runs through the same calls, the gradients of q, k and v meeting again in
the columns of one buffer.

    python examples/distill_step.py [--steps 5] [--dtype bf16|f32]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch  # noqa: E402

from mixed_step import NAMES, MixedStep  # noqa: E402

from paper_2607_28848_amd import attn, dsv, rope, vocab  # noqa: E402


class DistillStep(MixedStep):
    """MixedStep's block and batch with norms, rotation, a window and a teacher of `entries` logits a row.  A row's last
    token has no successor, so a sample's last row has no entries."""

    def __init__(self, requests, ranks, tokens, window=128, sinks=4, entries=8, temperature=2.0, theta=10000.0, **how):
        super().__init__(requests, ranks, tokens, **how)
        device, d = self.cache.device, self.head_dim
        gen = torch.Generator().manual_seed(how.get("seed", 0) + 1)
        self.window, self.sinks, self.temperature = window, sinks, temperature
        self.attn_plan = attn.Plan(self.seqs, self.n_rows, self.n_cache, self.heads_q, self.heads_kv, d, device=device,
                                   window=window, sinks=sinks)
        self.pos = torch.tensor([kl - ql + i for _, ql, _, kl, _ in self.seqs for i in range(ql)], dtype=torch.int32, device=device)
        self.slots = self.cache_rows.to(torch.int32)
        self.train_rows = self.train.to(torch.int32)
        self.freq = rope.frequencies(d, theta, device=device)
        self.q_norm, self.k_norm = ((1 + 0.1 * torch.randn(d, generator=gen)).to(device) for _ in range(2))
        n = len(self.train)
        ids = torch.randint(0, self.vocabulary, (n, entries), generator=gen, dtype=torch.int32)
        ids[:, 0] = torch.clamp(self.target[self.train].cpu(), min=0)  # the teacher likes the text's own token best
        self.teacher = torch.randn((n, entries), generator=gen).sort(1, descending=True).values.mul(2).to(device)
        self.ids = torch.where(self.target[self.train].cpu()[:, None] < 0, -1, ids).to(device)

    def _rope(self):
        return dict(q_weight=self.q_norm, k_weight=self.k_norm)

    def forward(self):
        X = self.embedding[self.tokens]
        qkv = torch.empty((self.n_rows, self.heads_q + 2 * self.heads_kv, self.head_dim), dtype=self.dtype, device=X.device)
        q, k, v = qkv.split([self.heads_q, self.heads_kv, self.heads_kv], dim=1)  # views: no copy joins the projections
        out = dsv.cobatch_fwd_grouped(self.plan, [(X, self.W[n], self.A[n], self.B[n], y) for n, y in zip(
            "qkv", qkv.flatten(1).split([self.nq, self.nkv, self.nkv], dim=1))])
        H = {n: h for n, (_, h) in zip("qkv", out)}
        Q, _, _ = rope.fwd(q, k, self.pos, self.freq, V=v, slots=self.slots, K_out=self.cache[0], V_out=self.cache[1],
                           **self._rope())
        O, lse = attn.fwd(self.attn_plan, Q, self.cache[0], self.cache[1])
        Z, H["o"] = dsv.cobatch_fwd(self.plan, O.flatten(1), self.W["o"], self.A["o"], self.B["o"])
        return X + Z, (X, q, k, Q, O, lse, H)

    def backward(self, hidden, saved):
        """The samples' mean loss, {projection: (dA, dB)} and the norm weights' gradients."""
        X, q, k, Q, O, lse, H = saved
        weight = (self.ids[:, 0] >= 0).float()
        weight /= weight.sum().clamp(min=1)
        loss, dZ = vocab.distill_grad(hidden[self.train], self.head, self.ids, self.teacher, temperature=self.temperature,
                                      weight=weight * self.temperature ** 2, Wt=self.head_t)
        grads = {"o": dsv.lora_bwd(self.plan, O.flatten(1), self.W["o"], self.A["o"], self.B["o"], H["o"], dZ)}
        dO = grads["o"][2].unflatten(1, (self.heads_q, self.head_dim))
        rows = torch.empty((len(self.train), self.heads_q + 2 * self.heads_kv, self.head_dim), dtype=self.dtype, device=X.device)
        dq, dk, dv = rows.split([self.heads_q, self.heads_kv, self.heads_kv], dim=1)
        attn.bwd(self.attn_plan, Q, self.cache[0], self.cache[1], O, lse, dO, dQ=dq, dK=dk, dV=dv)
        _, _, dq_norm, dk_norm = rope.bwd(dq, dk, self.pos, self.freq, rows=self.train_rows, Q=q, K=k, dQ_out=dq, dK_out=dk,
                                          want_weights=True, **self._rope())
        # the embedding is frozen: the block's input needs no gradient
        out = dsv.lora_bwd_grouped(self.plan, [(X, self.W[n], self.A[n], self.B[n], H[n], g) for n, g in zip(
            "qkv", rows.flatten(1).split([self.nq, self.nkv, self.nkv], dim=1))], want_dx=False)
        grads.update(zip("qkv", out))
        return (loss * weight).sum() * self.temperature ** 2, {n: grads[n][:2] for n in NAMES}, (dq_norm, dk_norm)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    # two prompts, one of them behind a cached prefix; decode tokens; two samples of adapter 0
    requests = [(0, 200, 1, 0), (300, 120, 2, 0)] + [(500 + 37 * i, 1, i % 4, 0) for i in range(6)] + \
        [(0, 256, 0, 1), (0, 100, 0, 1)]
    n = sum(r[1] for r in requests)
    tokens = torch.randint(0, 2000, (n,), generator=torch.Generator().manual_seed(1))
    block = DistillStep(requests, [16, 8, 32, 16], tokens, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    for i in range(a.steps):
        hidden, saved = block.forward()
        loss, grads, _ = block.backward(hidden, saved)
        block.update(grads)
        print("step %d: samples' mean divergence from the teacher %.4f" % (i + 1, float(loss)), flush=True)


if __name__ == "__main__":
    main()
