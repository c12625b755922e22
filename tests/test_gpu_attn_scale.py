"""Scales at the ends of fp32: refused where they or their multiple by log2 e are not positive and finite there, right
up to that."""
import pytest
import torch

from attn_util import check, oracle

pytestmark = pytest.mark.gpu
SEQS = [(0, 70, 0, 70, 1), (70, 1, 70, 90, 0)]


def tensors(dtype, q_std=1.0):
    g = torch.Generator().manual_seed(1)
    return [(torch.randn((n, h, 64), generator=g) * s).to(dtype).cuda() for n, h, s in ((71, 4, q_std), (160, 2, 1.0), (160, 2, 1.0))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_refused(dtype):
    from paper_2607_28848_amd import attn, dsv
    plan = attn.Plan(SEQS, 71, 160, 4, 2, 64, device="cuda")
    q, k, v = tensors(dtype)
    o, lse = attn.fwd(plan, q, k, v)
    for scale in (1e-50, 5e-46, 3e38, 2.36e38, 3.5e38):
        with pytest.raises(dsv.DsvError) as e:
            attn.fwd(plan, q, k, v, scale=scale)
        assert e.value.status == dsv.ERR_RANGE
        with pytest.raises(dsv.DsvError) as e:
            attn.bwd(plan, q, k, v, o, lse, o[:70], scale=scale)
        assert e.value.status == dsv.ERR_RANGE
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale,q_std", [(1e-42, 1.0), (1e-30, 1e28), (2e38, 1e-37)])
def test_accepted(dtype, scale, q_std):
    """Masked keys drop out at any of them."""
    from paper_2607_28848_amd import attn
    plan = attn.Plan(SEQS, 71, 160, 4, 2, 64, device="cuda")
    q, k, v = tensors(dtype, q_std)
    o, lse = attn.fwd(plan, q, k, v, scale=scale)
    want = oracle(SEQS, q, k, v, scale)
    check(o, want["O"], "O")
    check(lse, want["lse"], "lse")
