"""What the bindings of attention and the vocabulary loss refuse before the library is called (CPU only).  Each call
has a host-only plan or no workspace, which the library refuses as well (DsvError): nothing is ever launched."""
import types

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
