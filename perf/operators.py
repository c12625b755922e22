"""The operators between and after the co-batched linear layers: attention of a mixed batch, and the vocabulary loss.

``attn``   softmax attention of packed sequences of different lengths, causal, with grouped heads: whole prompts, chunks
           behind a cached prefix, single decode tokens over long caches, and the gradients of the fine-tuning samples.
``vocab``  softmax cross entropy of rows against a large vocabulary: the head's product, the loss and the gradient that
           reaches the rows (the head's weight is frozen), without logits kept for the whole vocabulary.

One case is one pass with the tensors, plan, workspace and outputs that a serving or fine-tuning program keeps.  Head
layouts and widths are those of the layers that this repository's workloads have (4096 wide: 32 heads on 8; 8192 wide:
64 on 8; heads of 128), and generic ones.

Fields of an attention case (op "attn"):
    what      "fwd" or "step" (forward, and backward of the fine-tuning samples)
    decode, ctx                  one-token sequences and the mean length of their caches
    chunk, chunk_len, prefix     chunks of a prompt, their length and the cached tokens before them
    prefill, prefill_len         whole prompts and their mean length
    train, train_len             fine-tuning samples and their length
    ragged                       log-normal lengths (else all alike)
    hq, hkv, d                   query heads, key / value heads, head width
    layout    "fused": K and V are columns of the rows that hold Q, as one q/k/v product leaves them
              "cache": K and V rows lie in slots of a cache, [row][head][d];  "heads": the same, [head][row][d]
    table     the number that the order and lengths are drawn from
Fields of a loss case (op "vocab"):
    what      "score" (losses alone) or "step" (losses and the gradient of the rows)
    T, K, V   rows, width, vocabulary;  wt: the transposed head is kept as well
Both: dtype "bf16" or "f32".
"""
import math
import random

import torch

own = False

ATTN = dict(op="attn", what="fwd", decode=0, ctx=0, chunk=0, chunk_len=0, prefix=0, prefill=0, prefill_len=0, train=0,
            train_len=0, ragged=False, hq=32, hkv=8, d=128, layout="cache", table=1, dtype="bf16")
VOCAB = dict(op="vocab", what="step", T=0, K=4096, V=128256, wt=False, dtype="bf16")


def listed():
    return [dict(base, name=name, **fields) for name, base, fields in (
        # A decode step of a small serving batch: eight tokens on caches of a few hundred rows, where latency counts.
        ("attn_decode8", ATTN, dict(decode=8, ctx=400, ragged=True, table=5)),
        # A decode step of a busy server: 64 tokens on caches of very different lengths, two to three thousand rows each.
        ("attn_decode64", ATTN, dict(decode=64, ctx=2600, ragged=True, table=7, layout="heads")),
        # A chunked-prefill step: 48 decode tokens beside a chunk of a long prompt whose first 5000 tokens are cached.
        ("attn_chunk365", ATTN, dict(decode=48, ctx=700, chunk=1, chunk_len=317, prefix=5003, ragged=True, table=9)),
        # Prompts of uneven length packed in one batch, narrow heads, inference only.
        ("attn_prefill_ragged_d64", ATTN, dict(prefill=9, prefill_len=700, ragged=True, hq=24, hkv=4, d=64,
                                               layout="fused", table=3)),
        # One whole long prompt.
        ("attn_prompt_16k", ATTN, dict(prefill=1, prefill_len=16384, layout="fused")),
        # The framework's flagship batch: eight prompts of 512 beside two fine-tuning samples of 1024, both directions.
        ("attn_mixed_8b_step", ATTN, dict(what="step", prefill=8, prefill_len=512, train=2, train_len=1024,
                                          layout="fused")),
        # Four fine-tuning samples of 2048 on the wider layer, both directions.
        ("attn_ft_70b_step", ATTN, dict(what="step", train=4, train_len=2048, hq=64, layout="fused")),
        # fp32, both directions, odd lengths (the smallest workload of the benchmark runs in fp32).
        ("attn_f32_step", ATTN, dict(what="step", prefill=2, prefill_len=96, train=3, train_len=157, hq=8, hkv=2, d=64,
                                     layout="fused", dtype="f32")),
        # The log-probability of one sampled token (scoring, speculative checks): the head is read once.
        ("vocab_score1", VOCAB, dict(what="score", T=1)),
        # The paper's 256 accumulated fine-tuning tokens: loss and gradient of the rows.
        ("vocab_ft256_step", VOCAB, dict(T=256, wt=True)),
        # Four fine-tuning samples of 1024 on the wider layer, without a transposed copy of the head.
        ("vocab_ft4096_70b_step", VOCAB, dict(T=4096, K=8192)),
        # fp32, odd rows, an odd vocabulary.
        ("vocab_f32_step", VOCAB, dict(T=333, K=512, V=5003, dtype="f32")),
    )]


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("decode", "decode", "chunk", "prefill", "step", "step", "f32", "score", "loss", "loss", "loss32"))
    if kind in ("score", "loss", "loss32"):
        c = dict(VOCAB, what="score" if kind == "score" else "step")
        if kind == "loss32":
            c.update(dtype="f32", T=log_int(5, 600), K=8 * log_int(8, 128), V=log_int(300, 20000), wt=rng.random() < 0.5)
            c["what"] = rng.choice(("score", "step"))
        else:
            c.update(T=log_int(1, 64) if kind == "score" else log_int(16, 2500), K=8 * log_int(64, 1024),
                     V=log_int(4000, 160000), wt=kind == "loss" and rng.random() < 0.5)
        return c
    c = dict(ATTN, table=rng.randrange(1, 1 << 20), ragged=rng.random() < 0.7)
    c["hkv"], group = rng.choice((1, 2, 4, 8, 8, 8)), rng.choice((1, 3, 4, 4, 7, 8))
    c["hq"], c["d"] = c["hkv"] * group, rng.choice((64, 128, 128))
    c["layout"] = rng.choice(("cache", "heads"))
    if kind == "decode":
        c.update(decode=log_int(1, 96), ctx=log_int(30, 6000))
    elif kind == "chunk":
        c.update(decode=rng.choice((0, log_int(1, 64))), ctx=log_int(30, 2000), chunk=rng.randint(1, 3),
                 chunk_len=log_int(2, 700), prefix=log_int(20, 6000))
    elif kind == "prefill":
        c.update(prefill=rng.randint(1, 12), prefill_len=log_int(20, 2500), layout=rng.choice(("fused", "cache")))
    elif kind == "step":
        c.update(what="step", prefill=rng.randint(0, 6), prefill_len=log_int(20, 1000), train=rng.randint(1, 4),
                 train_len=log_int(30, 2048), layout="fused")
    else:
        c.update(what=rng.choice(("fwd", "step")), prefill=rng.randint(0, 3), prefill_len=log_int(8, 200),
                 train=rng.randint(1, 3), train_len=log_int(16, 300), hkv=2, hq=2 * group, layout="fused", dtype="f32")
    return c


# ---- the batch ------------------------------------------------------------------------------------------------------
def table(case):
    """(sequences, rows of Q, rows of K and V): [(q_start, q_len, k_start, k_len, is_train)] in batch order.  Query i of
    a sequence sees its first k_len - q_len + i + 1 keys."""
    rng = random.Random(case["table"])

    def length(n):
        return max(1, min(3 * n, int(round(rng.lognormvariate(math.log(0.85 * n), 0.6))))) if case["ragged"] else n

    pieces = [(1, length(case["ctx"]), 0) for _ in range(case["decode"])]
    for _ in range(case["chunk"]):
        pieces.append((case["chunk_len"], case["chunk_len"] + length(case["prefix"]), 0))
    for _ in range(case["prefill"]):
        n = length(case["prefill_len"])
        pieces.append((n, n, 0))
    pieces += [(case["train_len"], case["train_len"], 1)] * case["train"]
    rng.shuffle(pieces)
    seqs, nq, nk = [], 0, 0
    for ql, kl, train in pieces:
        seqs.append((nq, ql, nq if case["layout"] == "fused" else nk, kl, train))
        nq += ql
        nk += kl + (-kl) % 64  # a slot of the cache: whole blocks of 64 rows
    return seqs, nq, nq if case["layout"] == "fused" else nk


def pairs(seqs):
    """(query, key) pairs that the causal mask leaves."""
    return sum(ql * kl - ql * (ql - 1) // 2 for _, ql, _, kl, _ in seqs)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "vocab":
        T, K, V = case["T"], case["K"], case["V"]
        step = case["what"] == "step"
        return {"flops": (4 if step else 2) * T * K * V, "bytes": (V * K + T * K * (2 if step else 1)) * size + 12 * T}
    seqs, _, _ = table(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    nq, nk = sum(s[1] for s in seqs), sum(s[3] for s in seqs)
    flops, moved = 4 * d * hq * pairs(seqs), 2 * (nq * hq + nk * hkv) * d * size
    if case["what"] == "step":  # scores again, dV, dP, dQ, dK; dO read, dQ, dK and dV written
        train = [s for s in seqs if s[4]]
        flops += 10 * d * hq * pairs(train)
        moved += sum(s[1] for s in train) * (2 * hq + 2 * hkv) * d * size
    return {"flops": flops, "bytes": moved}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    return _prepare_vocab(case, seed) if case["op"] == "vocab" else _prepare_attn(case, seed)


def run(st):
    if own:
        return _own_vocab(st) if st["case"]["op"] == "vocab" else _own_attn(st)
    return _plain_vocab(st) if st["case"]["op"] == "vocab" else _plain_attn(st)


def exact(case, seed):
    return _exact_vocab(case, seed) if case["op"] == "vocab" else _exact_attn(case, seed)


# ---- attention ------------------------------------------------------------------------------------------------------
def _prepare_attn(case, seed):
    """Queries twice as large as the keys: scores of standard deviation 2, so that rows are neither flat nor one-hot."""
    dev, dt = torch.device("cuda", torch.cuda.current_device()), _dtype(case)
    seqs, nq, nk = table(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    gen = torch.Generator(device=dev).manual_seed(1000003 * (seed % (1 << 30)) + case["table"])

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    st = dict(case=case, seqs=seqs, scale=1 / math.sqrt(d))
    if case["layout"] == "fused":
        rows = normal(nq, hq + 2 * hkv, d)
        rows[:, :hq] *= 2
        rows = rows.to(dt)
        st["Q"], st["K"], st["V"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    else:
        st["Q"] = (2 * normal(nq, hq, d)).to(dt)
        for name in ("K", "V"):
            if case["layout"] == "heads":
                st[name] = normal(hkv, nk, d).to(dt).transpose(0, 1)
            else:
                st[name] = normal(nk, hkv, d).to(dt)
    st["O"] = torch.empty((nq, hq, d), dtype=dt, device=dev)
    if case["what"] == "step":
        n = sum(s[1] for s in seqs if s[4])
        st["dO"] = normal(n, hq, d).to(dt)
        st["lse"] = torch.empty((hq, nq), dtype=torch.float32, device=dev)
        st["dQ"], st["dK"], st["dV"] = (torch.empty((n, h, d), dtype=dt, device=dev) for h in (hq, hkv, hkv))
    if own:
        from paper_2607_28848_amd import attn
        st["plan"] = attn.Plan(seqs, nq, nk, hq, hkv, d, device=dev)
        st["workspace"] = torch.empty(attn.workspace_bytes(st["plan"], _dtype(case)), dtype=torch.uint8, device=dev)
    return st


def _own_attn(st):
    from paper_2607_28848_amd import attn
    plan, ws = st["plan"], st["workspace"]
    if st["case"]["what"] == "fwd":
        attn.fwd(plan, st["Q"], st["K"], st["V"], scale=st["scale"], O=st["O"], workspace=ws)
        return st["O"]
    attn.fwd(plan, st["Q"], st["K"], st["V"], scale=st["scale"], O=st["O"], lse=st["lse"], workspace=ws)
    attn.bwd(plan, st["Q"], st["K"], st["V"], st["O"], st["lse"], st["dO"], scale=st["scale"], dQ=st["dQ"], dK=st["dK"],
             dV=st["dV"], workspace=ws)
    return st["O"], st["lse"], st["dQ"], st["dK"], st["dV"]


PLAIN_SCORES = 1 << 30  # scores held at once


def _visible(ql, kl, lo, hi, dev):
    """Keys that queries [lo, hi) of a sequence see."""
    return torch.arange(kl, device=dev)[None, :] <= torch.arange(lo, hi, device=dev)[:, None] + (kl - ql)


def _plain_attn(st):
    case, dev = st["case"], st["Q"].device
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, step = hq // hkv, case["what"] == "step"
    done = 0
    for q0, ql, k0, kl, train in st["seqs"]:
        # [hkv][group][ql][d] against [hkv][1][d][kl]
        q = st["Q"][q0:q0 + ql].float().reshape(ql, hkv, group, d).permute(1, 2, 0, 3)
        k = st["K"][k0:k0 + kl].float().permute(1, 0, 2).unsqueeze(1)
        v = st["V"][k0:k0 + kl].float().permute(1, 0, 2).unsqueeze(1)
        out = torch.empty((hkv, group, ql, d), device=dev)
        lse = torch.empty((hkv, group, ql), device=dev)
        rows = max(1, min(ql, PLAIN_SCORES // (hq * kl)))
        for lo in range(0, ql, rows):
            hi = min(ql, lo + rows)
            s = torch.matmul(q[:, :, lo:hi], k.transpose(-1, -2)) * st["scale"]
            s.masked_fill_(~_visible(ql, kl, lo, hi, dev), -math.inf)
            m = s.amax(dim=-1, keepdim=True)
            p = torch.exp(s - m)
            total = p.sum(dim=-1, keepdim=True)
            out[:, :, lo:hi] = torch.matmul(p, v) / total
            lse[:, :, lo:hi] = (m + torch.log(total)).squeeze(-1)
        st["O"][q0:q0 + ql] = out.permute(2, 0, 1, 3).reshape(ql, hq, d).to(st["O"].dtype)
        if not step:
            continue
        st["lse"][:, q0:q0 + ql] = lse.reshape(hq, ql)
        if not train:
            continue
        do = st["dO"][done:done + ql].float().reshape(ql, hkv, group, d).permute(1, 2, 0, 3)
        o = st["O"][q0:q0 + ql].float().reshape(ql, hkv, group, d).permute(1, 2, 0, 3)
        s = torch.matmul(q, k.transpose(-1, -2)) * st["scale"]
        s.masked_fill_(~_visible(ql, kl, 0, ql, dev), -math.inf)
        p = torch.exp(s - lse.unsqueeze(-1))
        dp = torch.matmul(do, v.transpose(-1, -2))
        ds = p * (dp - (do * o).sum(dim=-1, keepdim=True)) * st["scale"]
        dq = torch.matmul(ds, k)
        dk = torch.matmul(ds.transpose(-1, -2), q).sum(dim=1)
        dv = torch.matmul(p.transpose(-1, -2), do).sum(dim=1)
        st["dQ"][done:done + ql] = dq.permute(2, 0, 1, 3).reshape(ql, hq, d).to(st["dQ"].dtype)
        st["dK"][done:done + ql] = dk.permute(1, 0, 2).to(st["dK"].dtype)
        st["dV"][done:done + ql] = dv.permute(1, 0, 2).to(st["dV"].dtype)
        done += ql
    if not step:
        return st["O"]
    return st["O"], st["lse"], st["dQ"], st["dK"], st["dV"]


def _exact_attn(case, seed):
    """Head by head in 64 bits; the gradients from the softmax's own Jacobian, without the outputs."""
    if 14 * case["d"] * case["hq"] * sum(s[1] * s[3] for s in table(case)[0]) > 6e13:
        return None
    st = _prepare_attn(case, seed)
    hq, d, group = case["hq"], case["d"], case["hq"] // case["hkv"]
    step = case["what"] == "step"
    dev, f64 = st["Q"].device, torch.float64
    O = torch.zeros(st["O"].shape, dtype=f64, device=dev)
    lse = torch.zeros((hq, O.shape[0]), dtype=f64, device=dev)
    if step:
        dQ, dK, dV = (torch.zeros(st[n].shape, dtype=f64, device=dev) for n in ("dQ", "dK", "dV"))
    base = 0
    for q0, ql, k0, kl, train in st["seqs"]:
        for h in range(hq):
            g = h // group
            keys, values = st["K"][k0:k0 + kl, g].to(f64), st["V"][k0:k0 + kl, g].to(f64)
            for a in range(0, ql, 2048):
                b = min(ql, a + 2048)
                last = torch.arange(a, b, device=dev) + kl - ql  # the last key that each query sees
                x = st["Q"][q0 + a:q0 + b, h].to(f64) @ keys.t() * st["scale"]
                x = torch.where(torch.arange(kl, device=dev)[None, :] > last[:, None], x.new_tensor(-math.inf), x)
                norm = torch.logsumexp(x, dim=1)
                prob = torch.exp(x - norm[:, None])
                O[q0 + a:q0 + b, h], lse[h, q0 + a:q0 + b] = prob @ values, norm
                if step and train:
                    up = st["dO"][base + a:base + b, h].to(f64)
                    dV[base:base + kl, g] += prob.t() @ up
                    w = up @ values.t()
                    w = prob * (w - (prob * w).sum(dim=1, keepdim=True)) * st["scale"]
                    dQ[base + a:base + b, h] = w @ keys
                    dK[base:base + kl, g] += w.t() @ st["Q"][q0 + a:q0 + b, h].to(f64)
        base += ql if train else 0
    return (O, lse, dQ, dK, dV) if step else O


# ---- vocabulary loss ------------------------------------------------------------------------------------------------
def _prepare_vocab(case, seed):
    """Half of the rows lean to their target, as a trained model's do; a quarter of a sample's rows (the prompt's) have
    no target; the others weigh one over their number, the mean that a fine-tuning step takes."""
    dev, dt = torch.device("cuda", torch.cuda.current_device()), _dtype(case)
    T, K, V = case["T"], case["K"], case["V"]
    gen = torch.Generator(device=dev).manual_seed(1000003 * (seed % (1 << 30)) + 17)
    W = torch.empty((V, K), dtype=dt, device=dev)
    for lo in range(0, V, 16384):
        n = min(V, lo + 16384) - lo
        W[lo:lo + n] = torch.randn((n, K), generator=gen, device=dev) * (2 / math.sqrt(K))
    target = torch.randint(V, (T,), generator=gen, device=dev, dtype=torch.int32)
    X = torch.randn((T, K), generator=gen, device=dev)
    lean = torch.rand((T, 1), generator=gen, device=dev) < 0.5
    X += torch.where(lean, 3.0, 0.0) * W[target.long()].float()
    st = dict(case=case, X=X.to(dt), W=W, target=target, Wt=W.t().contiguous() if case["wt"] else None)
    if case["what"] == "step":
        st["target"] = target = torch.where(torch.arange(T, device=dev) % 4 == 1, -1, target).to(torch.int32)
        st["weight"] = torch.full((T,), 1 / max(1, T - (T + 2) // 4), dtype=torch.float32, device=dev)
        st["dX"] = torch.empty((T, K), dtype=dt, device=dev)
    st["loss"] = torch.empty((T,), dtype=torch.float32, device=dev)
    if own:
        from paper_2607_28848_amd import vocab
        st["workspace"] = torch.empty(vocab.workspace_bytes(T, K, V, dt, grad=case["what"] == "step"),
                                      dtype=torch.uint8, device=dev)
    return st


def _own_vocab(st):
    from paper_2607_28848_amd import vocab
    if st["case"]["what"] == "score":
        vocab.loss(st["X"], st["W"], st["target"], loss=st["loss"], workspace=st["workspace"])
        return st["loss"]
    vocab.loss_grad(st["X"], st["W"], st["target"], weight=st["weight"], Wt=st["Wt"], loss=st["loss"], dX=st["dX"],
                    workspace=st["workspace"])
    return st["loss"], st["dX"]


def _plain_vocab(st):
    rows = torch.arange(st["X"].shape[0], device=st["X"].device)
    W = st["W"].float()
    z = torch.matmul(st["X"].float(), W.t())
    m = z.amax(dim=1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(dim=1, keepdim=True)
    has = st["target"] >= 0
    t = st["target"].long().clamp(min=0)
    st["loss"].copy_(torch.where(has, torch.log(total[:, 0]) + m[:, 0] - z[rows, t], 0.0))
    if st["case"]["what"] == "score":
        return st["loss"]
    del z
    p /= total
    p[rows, t] -= 1
    p *= (st["weight"] * has)[:, None]
    st["dX"].copy_(torch.matmul(p, W).to(st["dX"].dtype))
    return st["loss"], st["dX"]


def _exact_vocab(case, seed):
    """Rows by rows in 64 bits; the gradient as the mean head row under the softmax, less the target's."""
    if case["T"] * case["K"] * case["V"] > 6e12:
        return None
    st = _prepare_vocab(case, seed)
    W = st["W"].to(torch.float64)
    loss, grad = [], []
    for lo in range(0, case["T"], 512):
        x, t = st["X"][lo:lo + 512].to(torch.float64), st["target"][lo:lo + 512].long()
        logp = torch.log_softmax(x @ W.t(), dim=1)
        keep = (t >= 0).to(torch.float64)
        at = t.clamp(min=0)
        loss.append(-logp.gather(1, at[:, None])[:, 0] * keep)
        if case["what"] == "step":
            prob = torch.exp(logp)
            prob.scatter_add_(1, at[:, None], torch.full_like(prob[:, :1], -1.0))
            grad.append(prob @ W * (st["weight"][lo:lo + 512].to(torch.float64) * keep)[:, None])
    return (torch.cat(loss), torch.cat(grad)) if case["what"] == "step" else torch.cat(loss)
