"""Attention of few heads and long rows, whose tiles run in pieces: forward tiles, the split form, dQ, dK and dV."""
import pytest
import torch

from test_gpu_attn import BF, place, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,layout", [(2, 1, 128, "cache"), (3, 3, 64, "heads"), (1, 1, 128, "padded"),
                                             (4, 1, 64, "fused")])
@pytest.mark.parametrize("lens", [[(1100, 1100, 1), (45, 45, 1)],              # one long sample, one short
                                  [(333, 1301, 1), (700, 650, 1), (1, 5, 1)],  # keys behind and short of the queries
                                  [(40, 2500, 0), (9, 3333, 0), (513, 513, 1)]])
def test_pieces(lens, hq, hkv, d, layout):
    print(lens, hq, hkv, d, layout, flush=True)
    seqs, nq, nk = place(lens, layout, q_gap=2)
    run(seqs, nq, nk, hq, hkv, d, BF, layout, seed=d + hq)


def test_pieces_repeat():
    """The pieces' sums are added in order: repeated calls give the same bits."""
    seqs, nq, nk = place([(900, 900, 1), (5, 2000, 0)], "cache")
    a, b = (run(seqs, nq, nk, 2, 1, 128, BF, "cache") for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)
