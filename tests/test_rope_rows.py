"""Gradient rows of a batch whose length nothing in the call states: without rotation and norm the rows' numbers bound nothing
(the library's entry is replaced by one that notes what it is given: nothing is launched)."""
import struct
import types

import pytest
import torch

from paper_2607_28848_amd import rope

STREAM = types.SimpleNamespace(cuda_stream=0)


@pytest.fixture
def given(monkeypatch):
    seen = []
    monkeypatch.setattr(torch.cuda, "is_available", lambda: False)  # the tensors are in host memory
    monkeypatch.setattr(rope, "_bwd", lambda dtype, r, n_rows, *rest: seen.append((struct.unpack_from("@i", r)[0], n_rows)) or 0)
    return seen


def test_rows_beyond_their_count_are_rows_of_the_batch(given):
    dQ = torch.randn((3, 4, 64))
    rope.bwd(dQ, None, None, None, rows=torch.tensor([0, 5, 9], dtype=torch.int32), dQ_out=torch.empty_like(dQ), stream=STREAM)
    (n, n_rows), = given
    assert n_rows == 3 and n > 9


def test_a_batch_that_is_stated_bounds_its_rows(given):
    dQ, out = torch.randn((3, 4, 64)), torch.empty((3, 4, 64))
    rows = torch.tensor([0, 5, 9], dtype=torch.int32)
    pos = torch.zeros(7, dtype=torch.int32)
    rope.bwd(dQ, None, pos, None, rows=rows, dQ_out=out, stream=STREAM)
    rope.bwd(dQ, None, None, None, rows=rows, Q=torch.zeros((8, 4, 64)), dQ_out=out, stream=STREAM)
    rope.bwd(dQ, None, None, None, dQ_out=out, stream=STREAM)
    assert given == [(7, 3), (8, 3), (3, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_without_rotation_and_norm_are_the_rows_themselves(dtype):
    gen = torch.Generator().manual_seed(2)
    dQ, dK = (torch.randn((5, h, 64), generator=gen).to(dtype).cuda() for h in (4, 2))
    rows = torch.tensor([0, 9, -1, 1 << 20, 3], dtype=torch.int32, device="cuda")
    for _ in range(2):
        a, b, none, none2 = rope.bwd(dQ, dK, None, None, rows=rows)
        torch.cuda.synchronize()
        assert none is None and none2 is None
        for x, y in ((a, dQ), (b, dK)):
            want = y.clone()
            want[2] = 0  # no row of any batch
            assert torch.equal(x, want)
    a, _, _, _ = rope.bwd(dQ, None, None, None)
    torch.cuda.synchronize()
    assert torch.equal(a, dQ)
