#!/usr/bin/env python3
"""One co-batched step through the linear layers, the attention and the vocabulary loss.

A batch holds new prompts, decode tokens behind cached prefixes and fine-tuning samples, each on its own LoRA adapter.
One forward serves all of them: q, k and v (grouped, into the columns of one buffer), the new keys and values into the
cache, attention over the cache, o.  The prompts' tokens are then scored, and the fine-tuning samples go back: the
vocabulary loss with the gradient of their last hidden rows, o, attention, q/k/v, AdamW.  Gradients hold the
fine-tuning rows alone, in the same order for every call, so each call's output is the next one's input.

The block is x + o(attention(q(x), k(x), v(x))) in front of the head: no norms, positions or MLP (gate, up and down are
three more linear layers, called like q, k and v).

    python examples/mixed_step.py [--steps 5] [--dtype bf16|f32]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2607_28848_amd import attn, dsv, vocab  # noqa: E402

NAMES = ("q", "k", "v", "o")


class MixedStep:
    """Weights, adapters, optimizer state and cache of one block, and the plans of one batch.

    requests: [(cached, new, adapter, is_train)] -- `new` rows behind `cached` rows of the cache; samples have no cached
    rows.  ranks: the adapters'.  tokens [T]: each row's token; a row's target is the token that follows it in the request.
    """

    def __init__(self, requests, ranks, tokens, heads_q=8, heads_kv=2, head_dim=64, vocabulary=2000,
                 dtype=torch.bfloat16, device="cuda", seed=0):
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, std=1.0, to=dtype):
            return (torch.randn(*shape, generator=gen) * std).to(device=device, dtype=to)

        hidden, r_max = heads_q * head_dim, max(ranks)
        self.hidden, self.vocabulary, self.dtype, self.ranks, self.r_max = hidden, vocabulary, dtype, list(ranks), r_max
        self.heads_q, self.heads_kv, self.head_dim = heads_q, heads_kv, head_dim
        self.nq, self.nkv = hidden, heads_kv * head_dim
        self.shapes = {"q": (hidden, self.nq), "k": (hidden, self.nkv), "v": (hidden, self.nkv), "o": (self.nq, hidden)}
        self.embedding = normal(vocabulary, hidden)
        self.head = normal(vocabulary, hidden, std=hidden ** -0.5)
        self.head_t = self.head.t().contiguous() if dtype == torch.bfloat16 else None
        self.W = {n: normal(N, K, std=K ** -0.5) for n, (K, N) in self.shapes.items()}
        self.A = {n: normal(len(ranks), r_max, K, std=K ** -0.5) for n, (K, N) in self.shapes.items()}
        self.B = {n: normal(len(ranks), N, r_max, std=0.02) for n, (K, N) in self.shapes.items()}
        self.state = {n: [t.float().clone() for t in (self.A[n], self.B[n])] +
                         [torch.zeros_like(t, dtype=torch.float32) for t in
                          (self.A[n], self.A[n], self.B[n], self.B[n])] for n in NAMES}
        self.steps = 0

        # rows of the batch and of the cache, request after request
        segments, seqs, rows, targets = [], [], [], []
        q0 = k0 = 0
        tokens = torch.as_tensor(tokens, dtype=torch.int64)
        for cached, new, adapter, is_train in requests:
            if is_train and cached:
                raise ValueError("a fine-tuning sample has no cached rows")
            segments.append((q0, new, adapter, int(is_train)))
            seqs.append((q0, new, k0, cached + new, int(is_train)))
            rows += range(k0 + cached, k0 + cached + new)
            targets += tokens[q0 + 1:q0 + new].tolist() + [-1] * min(new, 1)  # the last row has no target
            q0, k0 = q0 + new, k0 + cached + new
        self.segments, self.seqs, self.n_rows, self.n_cache = segments, seqs, q0, k0
        self.cache_rows = torch.tensor(rows, device=device)
        self.cache = torch.empty((2, k0, heads_kv, head_dim), dtype=dtype, device=device)
        for cached, new, k in zip([r[0] for r in requests], [r[1] for r in requests], [s[2] for s in seqs]):
            self.cache[:, k:k + cached] = normal(2, cached, heads_kv, head_dim)  # stands for earlier steps' rows
        self.tokens = tokens.to(device)
        self.target = torch.tensor(targets, dtype=torch.int32, device=device)
        self.plan = dsv.segments_build(segments, q0, ranks, [1.0] * len(ranks), r_max, device=device)
        self.attn_plan = attn.Plan(seqs, q0, k0, heads_q, heads_kv, head_dim, device=device)
        self.train = torch.from_numpy(self.plan.train_rows().copy()).long().to(device)
        train = set(self.train.tolist())
        self.scored = torch.tensor([i for i, t in enumerate(targets) if t >= 0 and i not in train], dtype=torch.int64,
                                   device=device)

    def forward(self):
        """Last hidden rows [T][hidden], and what the backward needs of them."""
        X = self.embedding[self.tokens]
        qkv = torch.empty((self.n_rows, self.nq + 2 * self.nkv), dtype=self.dtype, device=X.device)
        Y = dict(zip("qkv", qkv.split([self.nq, self.nkv, self.nkv], dim=1)))  # views: no copy joins the projections
        out = dsv.cobatch_fwd_grouped(self.plan, [(X, self.W[n], self.A[n], self.B[n], Y[n]) for n in "qkv"])
        H = {n: h for n, (_, h) in zip("qkv", out)}
        for cache, n in zip(self.cache, "kv"):
            cache[self.cache_rows] = Y[n].unflatten(1, (self.heads_kv, self.head_dim))
        O, lse = attn.fwd(self.attn_plan, Y["q"], self.cache[0], self.cache[1])
        Z, H["o"] = dsv.cobatch_fwd(self.plan, O.flatten(1), self.W["o"], self.A["o"], self.B["o"])
        return X + Z, (X, Y["q"], O, lse, H)

    def score(self, hidden):
        """-log p of the prompts' tokens, each given those before it."""
        return vocab.loss(hidden[self.scored], self.head, self.target[self.scored])

    def backward(self, hidden, saved):
        """The samples' mean loss and {projection: (dA, dB)}."""
        X, Q, O, lse, H = saved
        target = self.target[self.train]
        weight = (target >= 0).float()
        weight /= weight.sum().clamp(min=1)  # samples of one row have no target
        loss, dZ = vocab.loss_grad(hidden[self.train], self.head, target, weight=weight, Wt=self.head_t)
        grads = {}
        grads["o"] = dsv.lora_bwd(self.plan, O.flatten(1), self.W["o"], self.A["o"], self.B["o"], H["o"], dZ)
        dO = grads["o"][2].unflatten(1, (self.heads_q, self.head_dim))
        dY = attn.bwd(self.attn_plan, Q, self.cache[0], self.cache[1], O, lse, dO)
        # the embedding is frozen: the block's input needs no gradient
        out = dsv.lora_bwd_grouped(self.plan, [(X, self.W[n], self.A[n], self.B[n], H[n], g.flatten(1))
                                               for n, g in zip("qkv", dY)], want_dx=False)
        grads.update(zip("qkv", out))
        return (loss * weight).sum(), {n: grads[n][:2] for n in NAMES}

    def update(self, grads, lr=2e-3):
        self.steps += 1
        dsv.adamw_step_grouped(self.plan, self.steps, [(*grads[n], *self.state[n], self.A[n], self.B[n]) for n in NAMES],
                               lr=lr)


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
    block = MixedStep(requests, [16, 8, 32, 16], tokens, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    for i in range(a.steps):
        hidden, saved = block.forward()
        scores = block.score(hidden)
        loss, grads = block.backward(hidden, saved)
        block.update(grads)
        print("step %d: samples' mean loss %.4f, prompts' perplexity %.1f" % (
            i + 1, float(loss), math.exp(float(scores.mean()))), flush=True)


if __name__ == "__main__":
    main()
