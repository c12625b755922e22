"""Rows whose tiles take different references, both of weight: bringing one tile's terms to the other's must not round
them again."""
import pytest
import torch

from test_gpu_vocab import BF, F32, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", [1, -1])
def test_two_references(dtype, far):
    """Logits of 50 and about 51.4 in two tiles, more than 60 in base 2 from 0 (far = -1: below it, with all others
    lower still), where each tile takes a reference of its own.  The gradient's elements from 8 on come from one term
    alone, neither tile's largest, whose values lie where a rounding to bf16 is off the most: the bound has room for one."""
    T, K, V = 1500, 64, 1100
    g = torch.Generator().manual_seed(17)
    X, W = torch.zeros((T, K)), torch.zeros((V, K))
    X[:, 0] = 1
    X[:, 1] = -(0.69 + 0.01 * torch.rand(T, generator=g))
    X[:, 2] = 1.37 + 0.04 * torch.rand(T, generator=g)
    X[:, 3:5] = torch.rand((T, 2), generator=g)
    W[:, 0] = 0 if far > 0 else -75
    W[[100, 101, 700], 0] = 50.0 * far
    W[101, 1], W[101, 3], W[101, 8:] = 1, 2.0 ** -7, torch.rand((K - 8,), generator=g) * 0.1 + 1
    W[700, 2], W[700, 4] = 1, 2.0 ** -6
    target = torch.full((T,), 500, dtype=torch.int32)
    run(X.to(dtype).cuda(), W.to(dtype).cuda(), target.cuda(), None)
