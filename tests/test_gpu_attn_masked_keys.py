"""lse beside keys of -infinity scores and masked keys that hold NaN: of queries that do not see the NaN it is what it is
without either key."""
import math

import pytest
import torch

from attn_util import check, oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ql", [200, 9])
def test_lse_and_output(dtype, ql):
    from paper_2607_28848_amd import attn
    n, d, gone, nan = 200, 64, 20, 196
    g = torch.Generator().manual_seed(4)
    Q, K, V = (torch.randn((m, 2, d), generator=g).to(dtype) for m in (ql, n, n))
    Q[:, :, 0] = 1.0
    K[:gone, :, 0] = -math.inf
    K[nan, :, 1] = math.nan
    O, lse = attn.fwd(attn.Plan([(0, ql, 0, n, 0)], ql, n, 2, 2, d, device="cuda"), Q.cuda(), K.cuda(), V.cuda())
    free = ql - (n - nan)  # queries that do not see the NaN
    assert bool(O[free:].isnan().all()) and bool(lse[:, free:].isnan().all())
    K[:gone] = 0
    K[nan] = 0
    want = oracle([(0, free, gone, nan - gone, 0)], Q[:free], K, V, 1 / math.sqrt(d))
    check(O[:free], want["O"], "O")
    check(lse[:, :free], want["lse"], "lse")
