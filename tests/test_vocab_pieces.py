"""Widths of the vocabulary's pieces (CPU only), as the workspace shows them."""
import pytest
import torch

from paper_2607_28848_amd import vocab


@pytest.mark.parametrize("dtype,size,rows", [(torch.bfloat16, 2, 256), (torch.float32, 4, 64)])
@pytest.mark.parametrize("T", [1, 7, 15, 40])
@pytest.mark.parametrize("V", [1 << 20, (1 << 22) + 8, 1 << 23, 1 << 24])
def test_offsets_of_a_piece(dtype, size, rows, T, V):
    """The exponentials of a piece, [T][width], are addressed in 31 bits over a tile's rows, whether they exist or not.
    What else the workspace holds is taken from above, so `width` is at most a piece's."""
    K = 8
    ranges = 32 * T * K * 4 + 4 * 256  # at most: the second product's sums, rounded up
    rest = 4 * 4 * T + 256 + T * ((V + 63) // 64) * 8 + ranges
    width = (vocab.workspace_bytes(T, K, V, dtype, grad=True) - rest) // (T * size)
    assert rows * width * size < 1 << 31
