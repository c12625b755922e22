"""fp32 gradients behind a window: only long key tiles (the sinks') are summed in parts once the tiles fill the card, so the
workspace is the plain plan's and a little; and batches of whole and cut tiles side by side."""
import pytest
import torch

from paper_2607_28848_amd import attn

F32 = torch.float32


def bytes_of(lens, hq, hkv, d, **how):
    seqs, q = [], 0
    for n in lens:
        seqs.append((q, n, q, n, 1))
        q += n
    return attn.workspace_bytes(attn.Plan(seqs, q, q, hq, hkv, d, **how), F32)


@pytest.mark.parametrize("lens,hq,hkv,d,window", [([4096] * 8, 32, 8, 128, 256), ([2048] * 4, 32, 8, 128, 256), ([16384], 8, 2, 64, 64),
                                                  ([3000, 40, 9, 500], 16, 8, 64, 100)])
def test_workspace(lens, hq, hkv, d, window):
    plain = bytes_of(lens, hq, hkv, d)
    assert bytes_of(lens, hq, hkv, d, window=window) <= plain + 512 + (1 << 21)  # a sample's last tiles, which are short
    # and the sinks' tile of each sample: four parts of 16 rows of two gradients
    tile = hkv * 4 * 2 * 16 * d * 4
    assert bytes_of(lens, hq, hkv, d, window=window, sinks=4) <= plain + 512 + (1 << 21) + len(lens) * tile


def test_few_tiles_are_all_cut():
    """Under the number of CUs: 4 x 2 x 16 rows of each tile's, at most 16 MB."""
    assert bytes_of([357] * 3, 8, 2, 64, window=101) >= 3 * 23 * 2 * 4 * 2 * 16 * 64 * 4
    assert bytes_of([500] * 7, 8, 1, 128, window=101, sinks=3) <= 17 << 20


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[(700, 700, 1)], [(300, 300, 1), (40, 700, 1), (20, 20, 1), (513, 513, 1)], [(90, 90, 0), (600, 900, 1)]])
@pytest.mark.parametrize("window,sinks", [(64, 4), (33, 0), (16, 40), (250, 1)])
@pytest.mark.parametrize("hq,hkv,d", [(16, 8, 64), (8, 8, 128)])
def test_gradients_of_whole_and_cut_tiles(lens, window, sinks, hq, hkv, d):
    from test_gpu_attn import place
    from test_gpu_attn_window import run
    print(lens, window, sinks, hq, hkv, d, flush=True)
    run(*place(lens, "cache"), hq, hkv, d, F32, "cache", window, sinks, seed=7)
