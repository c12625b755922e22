"""The example's step with samples of one token each, none of which has a target: a loss of 0 and gradients of zeros."""
import pytest
import torch

from test_gpu_mixed_step import load

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_samples_without_a_target(dtype):
    tokens = torch.randint(0, 500, (42,), generator=torch.Generator().manual_seed(3))
    b = load().MixedStep([(0, 40, 1, 0), (0, 1, 0, 1), (0, 1, 1, 1)], [16, 8], tokens, heads_q=4, heads_kv=2, head_dim=64,
                         vocabulary=500, dtype=dtype)
    hidden, saved = b.forward()
    loss, grads = b.backward(hidden, saved)
    assert float(loss) == 0
    for dA, dB in grads.values():
        assert bool((dA == 0).all()) and bool((dB == 0).all())
