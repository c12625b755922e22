"""Operators around the attention and the loss of a co-batched step: what stands between the q/k/v products and the
attention, attention that looks back over a window, and the loss of a student that learns from a teacher.

``rope``  norms of queries and keys for each head and the position rotation, in one pass from the columns of the q/k/v
          product to the rows that the attention reads (queries, and keys and values in the slots of a cache), and the
          way back for the fine-tuning rows, with the norm weights' gradients.
``win``   softmax attention of packed sequences with a sliding window and a few first keys that stay visible: prompts,
          chunks behind a cached prefix, single tokens over long caches, and the gradients of the fine-tuning samples.
``kd``    the Kullback-Leibler divergence of the student's softmax over a large vocabulary from a teacher's top logits,
          with the gradient that reaches the rows (the head's weight is frozen).

Each case is one pass with the tensors, plan, workspace and outputs that a serving or fine-tuning program keeps.

Fields of a rotation case (op "rope"):
    what      "fwd" or "step" (forward of all rows, and backward of `train` of them)
    n, train  rows of the batch, fine-tuning rows
    hq, hkv, d, rot, pairs       heads, head width, rotated elements, "half" or "next" (which elements turn together)
    norm      whether queries and keys are normalised
    far       positions go up to this
Fields of an attention case (op "win"): those of a mixed batch's attention, and
    window, sinks                keys that a query looks back over (itself among them), first keys that stay visible
Fields of a distillation case (op "kd"):
    what      "score" (losses alone) or "step" (losses and the gradient of the rows)
    T, K, V, k                   rows, width, vocabulary, teacher's entries a row
    tau       temperature;  wt: the transposed head is kept as well
All: dtype "bf16" or "f32".
"""
import math
import random

import torch

own = False

ROPE = dict(op="rope", what="fwd", n=0, train=0, hq=32, hkv=8, d=128, rot=128, pairs="half", norm=True, far=8192,
            dtype="bf16")
WIN = dict(op="win", what="fwd", decode=0, ctx=0, chunk=0, chunk_len=0, prefix=0, prefill=0, prefill_len=0, train=0,
           train_len=0, ragged=False, hq=32, hkv=8, d=128, layout="cache", window=4096, sinks=4, table=1, dtype="bf16")
KD = dict(op="kd", what="step", T=0, K=4096, V=128256, k=32, tau=1.0, wt=False, dtype="bf16")


def listed():
    return [dict(base, name=name, **fields) for name, base, fields in (
        # A decode step of a small serving batch: eight tokens far into their texts, where latency counts.
        ("rope_decode8", ROPE, dict(n=8, far=100000)),
        # The framework's flagship batch: eight prompts of 512 beside two fine-tuning samples of 1024, both directions.
        ("rope_mixed_8b_step", ROPE, dict(what="step", n=6144, train=2048)),
        # A long prompt of the wider layer.
        ("rope_prompt_16k_70b", ROPE, dict(n=16384, hq=64, far=16384)),
        # fp32, both directions, odd rows, half of a head's elements turn, neighbours with neighbours.
        ("rope_f32_step", ROPE, dict(what="step", n=777, train=301, hq=8, hkv=2, d=64, rot=32, pairs="next",
                                     dtype="f32")),
        # A decode step of a busy server whose texts are three times as long as the window.
        ("win_decode64", WIN, dict(decode=64, ctx=12000, ragged=True, table=7, layout="heads")),
        # A chunked-prefill step: 24 decode tokens beside a chunk of a prompt whose first 30000 tokens are cached.
        ("win_chunk413", WIN, dict(decode=24, ctx=900, chunk=1, chunk_len=413, prefix=30000, ragged=True, table=9,
                                   window=2048, sinks=16)),
        # One whole long prompt.
        ("win_prompt_32k", WIN, dict(prefill=1, prefill_len=32768, layout="fused")),
        # Fine-tuning on long samples with a short window beside two prompts, both directions.
        ("win_ft_8k_step", WIN, dict(what="step", prefill=2, prefill_len=512, train=2, train_len=8192, layout="fused",
                                     window=1024)),
        # fp32, both directions, odd lengths, window and sinks.
        ("win_f32_step", WIN, dict(what="step", prefill=2, prefill_len=96, train=3, train_len=357, hq=8, hkv=2, d=64,
                                   layout="fused", window=101, sinks=3, dtype="f32")),
        # How far a student is from its teacher on a few held-out tokens: the head is read once.
        ("kd_score16", KD, dict(what="score", T=16, k=20)),
        # A fine-tuning sample of 1024 on the wider layer, softened, without a transposed copy of the head.
        ("kd_ft1024_70b_step", KD, dict(T=1024, K=8192, k=64, tau=2.0)),
        # fp32, odd rows, an odd vocabulary.
        ("kd_f32_step", KD, dict(T=333, K=512, V=5003, k=13, dtype="f32")),
    )]


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("rope", "rope", "rope", "decode", "chunk", "prefill", "train", "f32", "score", "loss", "loss",
                       "loss32"))
    if kind == "rope":
        c = dict(ROPE, what=rng.choice(("fwd", "step")), n=log_int(1, 16000), hkv=rng.choice((1, 2, 4, 8, 8)),
                 d=rng.choice((64, 128, 128)), pairs=rng.choice(("half", "half", "next")), norm=rng.random() < 0.75,
                 far=log_int(100, 1000000), dtype=rng.choice(("bf16", "bf16", "f32")))
        c["hq"] = c["hkv"] * rng.choice((1, 3, 4, 4, 7, 8))
        c["rot"] = rng.choice((c["d"], c["d"], c["d"] // 2, 16 * rng.randint(1, c["d"] // 16)))
        if c["what"] == "step":
            c["train"] = log_int(1, c["n"])
        return c
    if kind in ("score", "loss", "loss32"):
        c = dict(KD, what="score" if kind == "score" else "step", k=log_int(1, 100), tau=rng.choice((1.0, 1.0, 2.0, 3.5)))
        if kind == "loss32":
            c.update(dtype="f32", T=log_int(5, 600), K=8 * log_int(8, 128), V=log_int(300, 20000), wt=rng.random() < 0.5)
            c["what"] = rng.choice(("score", "step"))
        else:
            c.update(T=log_int(1, 64) if kind == "score" else log_int(16, 1200), K=8 * log_int(64, 800),
                     V=log_int(4000, 130000), wt=kind == "loss" and rng.random() < 0.5)
        return c
    c = dict(WIN, table=rng.randrange(1, 1 << 20), ragged=rng.random() < 0.7, window=log_int(16, 6000),
             sinks=rng.choice((0, 1, 4, 4, 16, 70, 128)))
    c["hkv"], group = rng.choice((1, 2, 4, 8, 8, 8)), rng.choice((1, 3, 4, 4, 7, 8))
    c["hq"], c["d"] = c["hkv"] * group, rng.choice((64, 128, 128))
    c["layout"] = rng.choice(("cache", "heads"))
    if kind == "decode":
        c.update(decode=log_int(1, 96), ctx=log_int(30, 15000))
    elif kind == "chunk":
        c.update(decode=rng.choice((0, log_int(1, 64))), ctx=log_int(30, 4000), chunk=rng.randint(1, 3),
                 chunk_len=log_int(2, 700), prefix=log_int(20, 20000))
    elif kind == "prefill":
        c.update(prefill=rng.randint(1, 8), prefill_len=log_int(20, 5000), layout=rng.choice(("fused", "cache")))
    elif kind == "train":
        c.update(what="step", prefill=rng.randint(0, 6), prefill_len=log_int(20, 1000), train=rng.randint(1, 4),
                 train_len=log_int(30, 3000), layout="fused")
    else:
        c.update(what=rng.choice(("fwd", "step")), prefill=rng.randint(0, 3), prefill_len=log_int(8, 200),
                 train=rng.randint(1, 3), train_len=log_int(16, 500), hkv=2, hq=2 * group, window=log_int(4, 300),
                 layout="fused", dtype="f32")
    return c


def prepare(case, seed):
    return {"rope": _prepare_rope, "win": _prepare_win, "kd": _prepare_kd}[case["op"]](case, seed)


def run(st):
    op = st["case"]["op"]
    if own:
        return {"rope": _own_rope, "win": _own_win, "kd": _own_kd}[op](st)
    return {"rope": _plain_rope, "win": _plain_win, "kd": _plain_kd}[op](st)


def exact(case, seed):
    return {"rope": _exact_rope, "win": _exact_win, "kd": _exact_kd}[case["op"]](case, seed)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        n, t, hq, hkv, d = case["n"], case["train"], case["hq"], case["hkv"], case["d"]
        # queries, keys and values read and written; gradients (and what the norms saw) read, gradients written
        moved = 2 * n * (hq + 2 * hkv) * d * size + 8 * n + t * (hq + hkv) * d * size * (3 if case["norm"] else 2)
        return {"flops": (n + t) * (hq + hkv) * d * (10 if case["norm"] else 4), "bytes": moved}
    if case["op"] == "kd":
        T, K, V, k = case["T"], case["K"], case["V"], case["k"]
        step = case["what"] == "step"
        return {"flops": (4 if step else 2) * T * K * V, "bytes": (V * K + T * K * (2 if step else 1)) * size + 8 * T * k + 8 * T}
    seqs, _, _ = table(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    nq = sum(s[1] for s in seqs)
    pairs = nk = both = 0
    for _, ql, _, kl, train in seqs:
        p, keys = _pairs(case, ql, kl)
        pairs, nk, both = pairs + p, nk + keys, both + (p if train else 0)
    flops, moved = 4 * d * hq * pairs, 2 * (nq * hq + nk * hkv) * d * size
    if case["what"] == "step":  # scores again, dV, dP, dQ, dK; dO read, dQ, dK and dV written
        flops += 10 * d * hq * both
        moved += sum(s[1] * 2 * hq + s[3] * 2 * hkv for s in seqs if s[4]) * d * size
    return {"flops": flops, "bytes": moved}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _device():
    return torch.device("cuda", torch.cuda.current_device())


# ---- norms and rotation -----------------------------------------------------------------------------------------------
EPS = 1e-6


def _prepare_rope(case, seed):
    """Rows of the fused product (queries and keys of different size from row to row), weights about 1, the slots of a
    cache in blocks of 16 rows, taken in any order."""
    dev, dt = _device(), _dtype(case)
    n, t, hq, hkv, d = case["n"], case["train"], case["hq"], case["hkv"], case["d"]
    gen = torch.Generator(device=dev).manual_seed(1000003 * (seed % (1 << 30)) + 29)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    rows = (normal(n, hq + 2 * hkv, d) * (0.5 + torch.rand((n, 1, 1), generator=gen, device=dev))).to(dt)
    blocks = (n + 15) // 16 + 3
    order = torch.randperm(blocks, generator=gen, device=dev)
    at = torch.arange(n, device=dev)
    st = dict(case=case, Q=rows[:, :hq], K=rows[:, hq:hq + hkv], V=rows[:, hq + hkv:],
              pos=torch.randint(case["far"], (n,), generator=gen, device=dev, dtype=torch.int32),
              freq=10000.0 ** (-torch.arange(0, case["rot"], 2, device=dev, dtype=torch.float64) / case["rot"]),
              slots=(16 * order[at // 16] + at % 16).to(torch.int32))
    st["q_weight"], st["k_weight"] = ((1 + 0.1 * normal(d)) if case["norm"] else None for _ in range(2))
    st["Q_out"] = torch.empty((n, hq, d), dtype=dt, device=dev)
    st["K_out"], st["V_out"] = (torch.zeros((16 * blocks, hkv, d), dtype=dt, device=dev) for _ in range(2))
    if case["what"] == "step":
        st["rows"] = torch.randperm(n, generator=gen, device=dev)[:t].sort().values.to(torch.int32)
        st["dQ"], st["dK"] = normal(t, hq, d).to(dt), normal(t, hkv, d).to(dt)
        out = torch.empty((t, hq + hkv, d), dtype=dt, device=dev)  # columns of the products' upstream gradient
        st["dQ_out"], st["dK_out"] = out[:, :hq], out[:, hq:]
        if case["norm"]:
            st["dq_weight"], st["dk_weight"] = (torch.empty((d,), device=dev) for _ in range(2))
        if own:
            from paper_2607_28848_amd import rope
            st["workspace"] = torch.empty(rope.workspace_bytes(t, hq, hkv, d), dtype=torch.uint8, device=dev)
    return st


def _own_rope(st):
    from paper_2607_28848_amd import rope
    case = st["case"]
    how = dict(q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, interleaved=case["pairs"] == "next")
    rope.fwd(st["Q"], st["K"], st["pos"], st["freq"], Q_out=st["Q_out"], K_out=st["K_out"], V=st["V"], V_out=st["V_out"],
             slots=st["slots"], **how)
    out = (st["Q_out"], st["K_out"], st["V_out"])
    if case["what"] == "fwd":
        return out
    kept = dict(Q=st["Q"], K=st["K"], dq_weight=st["dq_weight"], dk_weight=st["dk_weight"],
                workspace=st["workspace"]) if case["norm"] else {}
    rope.bwd(st["dQ"], st["dK"], st["pos"], st["freq"], rows=st["rows"], dQ_out=st["dQ_out"], dK_out=st["dK_out"], **how,
             **kept)
    return out + (st["dQ_out"], st["dK_out"]) + ((st["dq_weight"], st["dk_weight"]) if case["norm"] else ())


def _turn(case, pos, freq, back=False):
    """The rotation of [rows][heads][d] fp32 rows at these positions (angles in 64 bits), or its transpose."""
    angle = pos.double()[:, None] * freq[None, :]
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if back:
        s = -s
    half, rot = case["rot"] // 2, case["rot"]
    a, b = (slice(0, half), slice(half, rot)) if case["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))

    def turn(x):
        y = x.clone()
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        return y
    return turn


def _plain_rope(st):
    case = st["case"]
    dt, slots = st["Q"].dtype, st["slots"].long()

    def forward(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w
        return turn(x).to(dt)

    turn = _turn(case, st["pos"], st["freq"])
    st["Q_out"].copy_(forward(st["Q"], st["q_weight"]))
    st["K_out"][slots] = forward(st["K"], st["k_weight"])
    st["V_out"][slots] = st["V"]
    out = (st["Q_out"], st["K_out"], st["V_out"])
    if case["what"] == "fwd":
        return out
    rows = st["rows"].long()
    turn = _turn(case, st["pos"][rows], st["freq"], back=True)

    def backward(dy, x, w, to, dw):
        g = turn(dy.float())
        if w is not None:
            x = x[rows].float()
            r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
            unit = x * r
            dw.copy_((g * unit).double().sum(dim=(0, 1)))
            g = g * w
            g = r * (g - unit * (g * unit).mean(dim=-1, keepdim=True))
        to.copy_(g.to(dt))

    backward(st["dQ"], st["Q"], st["q_weight"], st["dQ_out"], st.get("dq_weight"))
    backward(st["dK"], st["K"], st["k_weight"], st["dK_out"], st.get("dk_weight"))
    return out + (st["dQ_out"], st["dK_out"]) + ((st["dq_weight"], st["dk_weight"]) if case["norm"] else ())


def _exact_rope(case, seed):
    """Pairs as complex numbers in 64 bits; the norm's gradient from its Jacobian."""
    st = _prepare_rope(case, seed)
    d, rot, half = case["d"], case["rot"], case["rot"] // 2
    turns = torch.polar(torch.ones_like(st["freq"])[None, :], torch.outer(st["pos"].to(torch.float64), st["freq"]))[:, None]

    def pairs(x):
        x = x[..., :rot]
        x = torch.stack((x[..., :half], x[..., half:]), -1) if case["pairs"] == "half" else x.unflatten(-1, (half, 2))
        return torch.view_as_complex(x.contiguous())

    def rotated(x, by):
        z = torch.view_as_real(pairs(x) * by)
        z = torch.cat((z[..., 0], z[..., 1]), -1) if case["pairs"] == "half" else z.flatten(-2)
        return torch.cat((z, x[..., rot:]), -1)

    def scaled(x, w):
        return x if w is None else w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS)

    slots = st["slots"].long()
    q, k = rotated(scaled(st["Q"].double(), st["q_weight"]), turns), rotated(scaled(st["K"].double(), st["k_weight"]), turns)
    K, V = (torch.zeros(st["K_out"].shape, dtype=torch.float64, device=q.device) for _ in range(2))
    K[slots], V[slots] = k, st["V"].double()
    if case["what"] == "fwd":
        return q, K, V
    rows, outs, dws = st["rows"].long(), [], []
    for name in ("Q", "K"):
        g = rotated(st["d" + name].double(), turns[rows].conj())
        w = st[name.lower() + "_weight"]
        if w is not None:
            x = st[name][rows].double()
            size2 = x.square().sum(-1, keepdim=True) / d + EPS
            dws.append((g * x / torch.sqrt(size2)).sum((0, 1)))
            g = g * w.double()
            g = g / torch.sqrt(size2) - x * ((g * x).sum(-1, keepdim=True) / (d * size2 ** 1.5))
        outs.append(g)
    return (q, K, V, *outs, *dws)


# ---- attention with a window and sinks --------------------------------------------------------------------------------
def table(case):
    """(sequences, rows of Q, rows of K and V): [(q_start, q_len, k_start, k_len, is_train)] in batch order.  Query i of
    a sequence stands at key k_len - q_len + i."""
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


def _pairs(case, ql, kl):
    """(query, key) pairs that the mask leaves, and the keys among them."""
    window, sinks = case["window"], case["sinks"]
    n = 0
    for p in range(kl - ql, kl):
        first = max(0, p + 1 - window)
        n += p + 1 - first + min(sinks, first)
    first = max(0, kl - ql + 1 - window)
    return n, kl - first + min(sinks, first)


def _prepare_win(case, seed):
    """Queries twice as large as the keys: scores of standard deviation 2, so that rows are neither flat nor one-hot."""
    dev, dt = _device(), _dtype(case)
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
        st["plan"] = attn.Plan(seqs, nq, nk, hq, hkv, d, device=dev, window=case["window"], sinks=case["sinks"])
        st["workspace"] = torch.empty(attn.workspace_bytes(st["plan"], _dtype(case)), dtype=torch.uint8, device=dev)
    return st


def _own_win(st):
    from paper_2607_28848_amd import attn
    plan, ws = st["plan"], st["workspace"]
    if st["case"]["what"] == "fwd":
        attn.fwd(plan, st["Q"], st["K"], st["V"], scale=st["scale"], O=st["O"], workspace=ws)
        return st["O"]
    attn.fwd(plan, st["Q"], st["K"], st["V"], scale=st["scale"], O=st["O"], lse=st["lse"], workspace=ws)
    attn.bwd(plan, st["Q"], st["K"], st["V"], st["O"], st["lse"], st["dO"], scale=st["scale"], dQ=st["dQ"], dK=st["dK"],
             dV=st["dV"], workspace=ws)
    return st["O"], st["lse"], st["dQ"], st["dK"], st["dV"]


def _plain_win(st):
    case, dev = st["case"], st["Q"].device
    hq, hkv, d, window, sinks = case["hq"], case["hkv"], case["d"], case["window"], case["sinks"]
    group, step, scale = hq // hkv, case["what"] == "step", st["scale"]
    done = 0
    for q0, ql, k0, kl, train in st["seqs"]:
        off = kl - ql
        # [hkv][group][ql][d] against [hkv][1][kl][d]
        q = st["Q"][q0:q0 + ql].float().reshape(ql, hkv, group, d).permute(1, 2, 0, 3)
        k = st["K"][k0:k0 + kl].float().permute(1, 0, 2).unsqueeze(1)
        v = st["V"][k0:k0 + kl].float().permute(1, 0, 2).unsqueeze(1)
        if step and train:
            do = st["dO"][done:done + ql].float().reshape(ql, hkv, group, d).permute(1, 2, 0, 3)
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        rows = max(128, min(1024, window))
        for lo in range(0, ql, rows):
            hi = min(ql, lo + rows)
            # the sinks, and the keys that some row of these looks back over
            first = max(0, lo + off + 1 - window)
            few = min(sinks, first)
            at = torch.cat((torch.arange(few, device=dev), torch.arange(first, hi + off, device=dev)))
            p = torch.arange(lo, hi, device=dev)[:, None] + off
            hidden = (at > p) | ((at + window <= p) & (at >= sinks))

            def part(x):
                return torch.cat((x[:, :, :few], x[:, :, first:hi + off]), dim=2)

            kp, vp = part(k), part(v)
            s = torch.matmul(q[:, :, lo:hi], kp.transpose(-1, -2)) * scale
            s.masked_fill_(hidden, -math.inf)
            m = s.amax(dim=-1, keepdim=True)
            s = torch.exp(s - m)
            total = s.sum(dim=-1, keepdim=True)
            s /= total
            out = torch.matmul(s, vp)
            st["O"][q0 + lo:q0 + hi] = out.permute(2, 0, 1, 3).reshape(hi - lo, hq, d).to(st["O"].dtype)
            if not step:
                continue
            st["lse"][:, q0 + lo:q0 + hi] = (m + torch.log(total)).reshape(hq, hi - lo)
            if not train:
                continue
            up = do[:, :, lo:hi]
            ds = s * (torch.matmul(up, vp.transpose(-1, -2)) - (up * out).sum(dim=-1, keepdim=True)) * scale
            dq = torch.matmul(ds, kp)
            st["dQ"][done + lo:done + hi] = dq.permute(2, 0, 1, 3).reshape(hi - lo, hq, d).to(st["dQ"].dtype)
            for to, x in ((dk, torch.matmul(ds.transpose(-1, -2), q[:, :, lo:hi])),
                          (dv, torch.matmul(s.transpose(-1, -2), up))):
                x = x.sum(dim=1, keepdim=True)
                to[:, :, :few] += x[:, :, :few]
                to[:, :, first:hi + off] += x[:, :, few:]
        if step and train:
            st["dK"][done:done + ql] = dk[:, 0].permute(1, 0, 2).to(st["dK"].dtype)
            st["dV"][done:done + ql] = dv[:, 0].permute(1, 0, 2).to(st["dV"].dtype)
            done += ql
    if not step:
        return st["O"]
    return st["O"], st["lse"], st["dQ"], st["dK"], st["dV"]


def _exact_win(case, seed):
    """Head by head in 64 bits, the rows' keys from a block of 256 on; the gradients from the softmax's own Jacobian."""
    seqs = table(case)[0]
    if 14 * case["d"] * case["hq"] * sum(_pairs(case, s[1], s[3])[0] + 2048 * s[1] for s in seqs) > 4e13:
        return None
    st = _prepare_win(case, seed)
    hq, d, group, window, sinks = case["hq"], case["d"], case["hq"] // case["hkv"], case["window"], case["sinks"]
    step = case["what"] == "step"
    dev, f64 = st["Q"].device, torch.float64
    O = torch.zeros(st["O"].shape, dtype=f64, device=dev)
    lse = torch.zeros((hq, O.shape[0]), dtype=f64, device=dev)
    if step:
        dQ, dK, dV = (torch.zeros(st[n].shape, dtype=f64, device=dev) for n in ("dQ", "dK", "dV"))
    base = 0
    for q0, ql, k0, kl, train in st["seqs"]:
        for a in range(0, ql, 2048):
            b = min(ql, a + 2048)
            pos = torch.arange(a, b, device=dev)[:, None] + (kl - ql)
            begin = max(0, a + kl - ql + 1 - window) // 256 * 256
            j = torch.arange(begin, b + kl - ql, device=dev)
            j = torch.cat((torch.arange(min(sinks, begin), device=dev), j))  # every key once
            seen = (j <= pos) & ((pos - j < window) | (j < sinks))
            for h in range(hq):
                g = h // group
                keys, values = st["K"][k0 + j, g].to(f64), st["V"][k0 + j, g].to(f64)
                x = st["Q"][q0 + a:q0 + b, h].to(f64) @ keys.t() * st["scale"]
                x = torch.where(seen, x, x.new_tensor(-math.inf))
                norm = torch.logsumexp(x, dim=1)
                prob = torch.exp(x - norm[:, None])
                O[q0 + a:q0 + b, h], lse[h, q0 + a:q0 + b] = prob @ values, norm
                if step and train:
                    up = st["dO"][base + a:base + b, h].to(f64)
                    dV[base:, g].index_add_(0, j, prob.t() @ up)
                    w = up @ values.t()
                    w = prob * (w - (prob * w).sum(dim=1, keepdim=True)) * st["scale"]
                    dQ[base + a:base + b, h] = w @ keys
                    dK[base:, g].index_add_(0, j, w.t() @ st["Q"][q0 + a:q0 + b, h].to(f64))
        base += ql if train else 0
    return (O, lse, dQ, dK, dV) if step else O


# ---- distillation -----------------------------------------------------------------------------------------------------
def _prepare_kd(case, seed):
    """The teacher's logits fall off from a row's first entry on, and the student leans to the first two; some rows have
    fewer entries than others, and a quarter of a sample's rows (the prompt's) none; the others weigh one over their
    number."""
    dev, dt = _device(), _dtype(case)
    T, K, V, k = case["T"], case["K"], case["V"], case["k"]
    gen = torch.Generator(device=dev).manual_seed(1000003 * (seed % (1 << 30)) + 43)
    W = torch.empty((V, K), dtype=dt, device=dev)
    for lo in range(0, V, 16384):
        n = min(V, lo + 16384) - lo
        W[lo:lo + n] = torch.randn((n, K), generator=gen, device=dev) * (2 / math.sqrt(K))
    ids = torch.randint(V, (T, k), generator=gen, device=dev)
    X = torch.randn((T, K), generator=gen, device=dev) + 2.5 * W[ids[:, 0]].float()
    if k > 1:
        X += 1.5 * W[ids[:, 1]].float()
    teacher = torch.randn((T, k), generator=gen, device=dev) + 8 - 3 * torch.log2(1.0 + torch.arange(k, device=dev))
    fewer = torch.randint(2 * k, (T, 1), generator=gen, device=dev).clamp(min=1)
    at = torch.arange(T, device=dev)[:, None]
    ids = torch.where((torch.arange(k, device=dev) >= fewer) | (at % 4 == 1), -1, ids)
    st = dict(case=case, X=X.to(dt), W=W, ids=ids.to(torch.int32), teacher=teacher, Wt=W.t().contiguous() if case["wt"] else None)
    st["loss"] = torch.empty((T,), dtype=torch.float32, device=dev)
    if case["what"] == "step":
        st["weight"] = torch.full((T,), case["tau"] ** 2 / max(1, T - (T + 2) // 4), dtype=torch.float32, device=dev)
        st["dX"] = torch.empty((T, K), dtype=dt, device=dev)
    if own:
        from paper_2607_28848_amd import vocab
        st["workspace"] = torch.empty(vocab.distill_workspace_bytes(T, K, V, k, dt, grad=case["what"] == "step"),
                                      dtype=torch.uint8, device=dev)
    return st


def _own_kd(st):
    from paper_2607_28848_amd import vocab
    case = st["case"]
    if case["what"] == "score":
        vocab.distill(st["X"], st["W"], st["ids"], st["teacher"], temperature=case["tau"], loss=st["loss"],
                      workspace=st["workspace"])
        return st["loss"]
    vocab.distill_grad(st["X"], st["W"], st["ids"], st["teacher"], temperature=case["tau"], weight=st["weight"],
                       Wt=st["Wt"], loss=st["loss"], dX=st["dX"], workspace=st["workspace"])
    return st["loss"], st["dX"]


def _plain_kd(st):
    tau = st["case"]["tau"]
    W = st["W"].float()
    z = torch.matmul(st["X"].float(), W.t())
    z /= tau
    m = z.amax(dim=1, keepdim=True)
    has = st["ids"] >= 0
    at = st["ids"].long().clamp(min=0)
    t = torch.where(has, st["teacher"] / tau, -math.inf)
    top = t.amax(dim=1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    q = torch.exp(t - top)
    mass = q.sum(dim=1, keepdim=True)
    some = mass > 0
    mass = torch.where(some, mass, 1.0)
    q = q / mass
    picked = z.gather(1, at)
    z -= m
    z.exp_()
    total = z.sum(dim=1, keepdim=True)
    terms = q * (t - top - torch.log(mass) - (picked - m - torch.log(total)))
    st["loss"].copy_(torch.where(q > 0, terms, 0.0).sum(dim=1))
    if st["case"]["what"] == "score":
        return st["loss"]
    z /= total
    z.scatter_add_(1, at, -q)
    z *= torch.where(some, st["weight"][:, None] / tau, 0.0)
    st["dX"].copy_(torch.matmul(z, W).to(st["dX"].dtype))
    return st["loss"], st["dX"]


def _exact_kd(case, seed):
    """Rows by rows in 64 bits, the teacher's entries spread over the vocabulary; the gradient as the difference of two
    mean head rows."""
    if case["T"] * case["K"] * case["V"] > 6e12:
        return None
    st = _prepare_kd(case, seed)
    f64, tau, V = torch.float64, case["tau"], case["V"]
    W = st["W"].to(f64)
    loss, grad = [], []
    for lo in range(0, case["T"], 256):
        x, ids = st["X"][lo:lo + 256].to(f64), st["ids"][lo:lo + 256].long()
        logp = torch.log_softmax(x @ W.t() / tau, dim=1)
        keep = ids >= 0
        some = keep.any(dim=1)
        t = (st["teacher"][lo:lo + 256].to(f64) / tau).masked_fill(~keep, -math.inf).masked_fill(~some[:, None], 0.0)
        logq = torch.log_softmax(t, dim=1)
        q = torch.exp(logq) * keep
        loss.append((q * (torch.where(keep, logq, 0.0) - torch.where(keep, logp.gather(1, ids.clamp(min=0)), 0.0))).sum(dim=1))
        if case["what"] == "step":
            full = torch.zeros((x.shape[0], V), dtype=f64, device=x.device).scatter_add_(1, ids.clamp(min=0), q)
            f = st["weight"][lo:lo + 256].to(f64) * some / tau
            grad.append((torch.exp(logp) @ W - full @ W) * f[:, None])
    return (torch.cat(loss), torch.cat(grad)) if case["what"] == "step" else torch.cat(loss)
