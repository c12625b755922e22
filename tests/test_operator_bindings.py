"""What the bindings of attention and the vocabulary loss refuse before the library is called (CPU only).  Each call
has a host-only plan or no workspace, which the library refuses as well (DsvError): nothing is ever launched."""
import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2607_28848_amd import attn, dsv, vocab

NONE = dict(workspace=torch.zeros(0, dtype=torch.uint8), stream=types.SimpleNamespace(cuda_stream=0))


def attention(back=False, **changed):
    p = attn.Plan([(0, 10, 0, 12, 1)], 10, 12, 4, 2, 64)
    t = dict(Q=torch.zeros((10, 4, 64)), K=torch.zeros((12, 2, 64)), V=torch.zeros((12, 2, 64)), O=torch.zeros((10, 4, 64)),
             lse=torch.zeros((4, 10)))
    if back:
        t.update(dO=torch.zeros((10, 4, 64)), dQ=torch.zeros((10, 4, 64)), dK=torch.zeros((12, 2, 64)),
                 dV=torch.zeros((12, 2, 64)))
    t.update(changed)
    return (attn.bwd if back else attn.fwd)(p, **NONE, **t)


def loss(grad=True, **changed):
    t = dict(X=torch.zeros((6, 16)), W=torch.zeros((8, 16)), target=torch.zeros(6, dtype=torch.int32), loss=torch.zeros(6))
    if grad:
        t.update(dX=torch.zeros((6, 16)))
    t.update(changed)
    return (vocab.loss_grad if grad else vocab.loss)(**NONE, **t)


def test_the_calls_as_they_are_reach_the_library():
    for call in (attention, lambda: attention(True), loss, lambda: loss(False)):
        with pytest.raises(dsv.DsvError):
            call()


@pytest.mark.parametrize("name,rows,heads", [("Q", 10, 4), ("K", 12, 2), ("V", 12, 2), ("O", 10, 4), ("dO", 10, 4),
                                             ("dQ", 10, 4), ("dK", 12, 2), ("dV", 12, 2)])
def test_broadcast_rows_and_heads_of_attention(name, rows, heads):
    """A stride of 0 stands for the dense one in the library: a broadcast tensor's would send it past its memory."""
    for t in (torch.zeros((rows, 1, 64)).expand(rows, heads, 64), torch.zeros((1, heads, 64)).expand(rows, heads, 64),
              torch.zeros((1, heads * 64)).expand(rows, heads * 64)):
        with pytest.raises(ValueError):
            attention(name in ("dO", "dQ", "dK", "dV"), **{name: t})


def test_broadcast_rows_of_the_loss():
    for name, rows, cols in (("X", 6, 16), ("W", 8, 16), ("dX", 6, 16), ("Wt", 16, 8)):
        with pytest.raises(ValueError):
            loss(**{name: torch.zeros((1, cols)).expand(rows, cols)})
    for name, rows in (("X", 6), ("W", 8)):
        with pytest.raises(ValueError):
            loss(False, **{name: torch.zeros((1, 16)).expand(rows, 16)})


def test_strides_of_single_rows_and_heads_are_free():
    p = attn.Plan([(0, 1, 0, 1, 0)], 1, 1, 1, 1, 64)
    t = torch.zeros((1, 1, 64)).as_strided((1, 1, 64), (0, 0, 1))
    with pytest.raises(dsv.DsvError):
        attn.fwd(p, t, t, t, O=t, **NONE)
    with pytest.raises(dsv.DsvError):
        loss(X=torch.zeros((1, 16)).as_strided((1, 16), (0, 1)), target=torch.zeros(1, dtype=torch.int32), loss=torch.zeros(1),
             dX=torch.zeros((1, 16)))


def far(rows, cols, row):
    return torch.empty_strided((rows, cols), (row, 1), dtype=torch.float32, device="meta")


def test_sizes_and_strides_past_32_bits():
    """The library takes them as 32-bit numbers: what does not fit is refused, not cut off."""
    big = 1 << 32
    for changed in (dict(X=far(6, 16, big + 16)), dict(W=far(8, 16, big + 16)), dict(dX=far(6, 16, big + 16)),
                    dict(Wt=far(16, 8, big + 8)), dict(X=far(big + 6, 16, 16), dX=far(big + 6, 16, 16)),
                    dict(W=far(big + 8, 16, 16)), dict(X=far(6, big + 16, big + 16), W=far(8, big + 16, big + 16),
                                                       dX=far(6, big + 16, big + 16))):
        with pytest.raises(ValueError):
            loss(**changed)
    for sizes in ((big + 6, 16, 8), (6, big + 16, 8), (6, 16, big + 8)):
        with pytest.raises(ValueError):
            vocab.workspace_bytes(*sizes, torch.float32, grad=True)
    with pytest.raises(ValueError):
        vocab.workspace_bytes(6, 16, 8, torch.float32, grad=True, ldw=big + 16)


def test_plans_past_32_bits():
    big = 1 << 32
    good = dict(seqs=[(0, 10, 0, 12, 1)], n_q=10, n_kv=12, heads_q=4, heads_kv=2, head_dim=64)
    attn.Plan(**good)
    attn.Plan(**dict(good, seqs=np.asarray(good["seqs"], np.int64)))
    for name, x in (("n_q", 10), ("n_kv", 12), ("heads_q", 4), ("heads_kv", 2), ("head_dim", 64)):
        with pytest.raises(ValueError):
            attn.Plan(**dict(good, **{name: big + x}))
    for i in range(5):
        for kind in (np.int64, np.uint32, float):
            s = np.asarray(good["seqs"], kind)
            s[0, i] += 1 << 31 if kind is np.uint32 else big
            with pytest.raises(ValueError):
                attn.Plan(**dict(good, seqs=s))


def test_broadcast_rows_of_the_grouped_linear_calls():
    p = dsv.segments_build([(0, 6, 0, 1)], 6, [8], [1.0], 8)
    t = dict(X=torch.zeros((6, 64)), W=torch.zeros((32, 64)), A=torch.zeros((1, 8, 64)), B=torch.zeros((1, 32, 8)))
    fwd = dict(t, Y=torch.zeros((6, 32)))
    bwd = dict(t, H=torch.zeros((6, 8)), dY=torch.zeros((6, 32)))
    with pytest.raises(dsv.DsvError):
        dsv.cobatch_fwd_grouped(p, [tuple(fwd.values())], **NONE)
    with pytest.raises(dsv.DsvError):
        dsv.lora_bwd_grouped(p, [tuple(bwd.values())], **NONE)
    for call, args, names in ((dsv.cobatch_fwd_grouped, fwd, ("X", "W", "Y")), (dsv.lora_bwd_grouped, bwd, ("X", "W", "dY"))):
        for name in names:
            rows, cols = args[name].shape
            bad = dict(args, **{name: torch.zeros((1, cols)).expand(rows, cols)})
            with pytest.raises(ValueError):
                call(p, [tuple(bad.values())], **NONE)


def test_backward_without_the_forwards_lse():
    """Refused by name where the plan has fine-tuning samples, else a no-op as in the library, which reads none then."""
    with pytest.raises(ValueError, match="lse"):
        attention(True, lse=None)
    p = attn.Plan([(0, 10, 0, 12, 0)], 10, 12, 4, 2, 64)
    q, k, none = torch.zeros((10, 4, 64)), torch.zeros((12, 2, 64)), torch.zeros((0, 4, 64))
    with pytest.raises(dsv.DsvError):  # it reaches the library: the plan is on the host
        attn.bwd(p, q, k, k, q, None, none, **NONE)


def test_lse_is_made_where_it_is_wanted():
    """As shown by where the call would make it: on a device of its own making, here the host."""
    made = []
    p = attn.Plan([(0, 10, 0, 12, 1)], 10, 12, 4, 2, 64)
    full = torch.full

    def record(*a, **kw):
        made.append(a[0])
        return full(*a, **kw)

    q, k = torch.zeros((10, 4, 64)), torch.zeros((12, 2, 64))
    lse = torch.zeros((4, 10))
    for kw, n in ((dict(), 1), (dict(O=q), 0), (dict(O=q, want_lse=True), 1), (dict(want_lse=True), 1), (dict(want_lse=False), 0),
                  (dict(O=q, want_lse=False), 0), (dict(lse=lse), 0), (dict(O=q, lse=lse, want_lse=True), 0)):
        made.clear()
        with pytest.MonkeyPatch.context() as m:
            m.setattr(torch, "full", record)
            m.setattr(attn, "on", lambda stream: contextlib.nullcontext())
            with pytest.raises(dsv.DsvError):
                attn.fwd(p, q, k, k, **kw, **NONE)
        assert made == [(4, 10)] * n, kw
