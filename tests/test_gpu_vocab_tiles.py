"""The vocabulary loss at sizes that take each of its tiles on a card of 256 CUs, with odd rows and columns, contractions
that end inside a step, vocabularies that end inside a tile, and a target in the last column."""
import pytest
import torch

from test_gpu_vocab import BF, F32, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,T,K,V", [
    (BF, 100, 72, 33001),   # 128 x 256 tiles
    (BF, 100, 192, 33024),
    (BF, 130, 200, 33003),  # 256 x 256
    (BF, 257, 64, 70001),   # two row tiles
    (BF, 190, 264, 20001),  # 128 x 128
    (BF, 600, 8, 5003),
    (BF, 600, 448, 5120),
    (BF, 65, 1000, 9001),   # 64 x 64, more rows than one tile
    (BF, 2, 64, 16385),
    (BF, 31, 456, 6001),
    (F32, 21, 328, 40001),  # 32 x 128, several rounds
    (F32, 97, 40, 33001),   # 64 x 128
    (F32, 33, 100 * 8, 130),
])
def test_tiles(dtype, T, K, V):
    print(dtype, T, K, V, flush=True)
    X, W, target, weight = make(T, K, V, dtype, seed=T)
    target[0] = V - 1
    run(X, W, target, weight)
    if dtype == BF:
        run(X, W, target, weight, Wt=W.t().contiguous())
