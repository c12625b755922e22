"""A plan with a window and sinks, which is built for every batch, takes the host little more than one without (CPU only)."""
import time

import pytest

from paper_2607_28848_amd import attn


def least(seqs, n, **how):
    best = float("inf")
    for _ in range(12):
        start = time.perf_counter()
        attn.Plan(seqs, n, n, 32, 8, 128, **how)
        best = min(best, time.perf_counter() - start)
    return best


@pytest.mark.parametrize("length,samples,window", [(16384, 8, 64), (131072, 1, 512), (8192, 4, 1024)])
def test_build(length, samples, window):
    seqs, n = [(i * length, length, i * length, length, 1) for i in range(samples)], samples * length
    plain, behind = least(seqs, n), least(seqs, n, window=window, sinks=4)
    # 1.1 to 1.3 times; 5 to 7 where every schedule that is tried takes its pieces one by one
    assert behind < 3 * plain, (plain, behind)
