"""Cosines and sines of far positions and fast frequencies against exactly reduced angles.

A head that is (1, 0) in every pair turns into its pairs' cosines and sines.  With e = 2^-24 and t the reduced angle, at most
pi / 4: t is rounded to fp32 once, 0.79 e; sin t = t + t^3 P takes six roundings of t^3 P <= 0.081 and one of at most 0.71,
cos t = 1 + t^2 Q five of t^2 Q <= 0.30 and one of 1, and the series end below 0.1 e.  So either is off by at most
0.79 e + 0.49 e + 0.71 e + 0.1 e or 0.56 e + 1.5 e + e + 0.1 e: 4 e covers both."""
import math
from decimal import Decimal, getcontext

import pytest
import torch

pytestmark = pytest.mark.gpu
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def exact(pos, freq):
    getcontext().prec = 60
    angle = Decimal(pos) * Decimal(freq)  # both exactly
    angle = float(angle - 2 * PI * (angle / (2 * PI)).to_integral_value())
    return math.cos(angle), math.sin(angle)


@pytest.mark.parametrize("interleaved", [False, True])
def test_cosines_and_sines(interleaved):
    from paper_2607_28848_amd import rope
    where = [0, 1, -1, 7, 5000, (1 << 24) + 1, 123456789, -987654321, (1 << 31) - 1, (1 << 31) - 2, -(1 << 31)]
    freq = [1.0, 0.75, 10000.0 ** (-1 / 64), 3.0, math.pi / 2, math.pi, 10.0, 1000.0, 1e6, 1e-3, 1e-12, 0.0, 2.5, 6.25, 100.0, 31.0]
    pos = torch.tensor(where, dtype=torch.int32, device="cuda")
    x = torch.zeros((len(where), 1, 64), device="cuda")
    first, second = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
    x[:, :, first] = 1.0
    y, _ = rope.fwd(x, None, pos, torch.tensor(freq, dtype=torch.float64, device="cuda"), interleaved=interleaved)
    # and the other way: the backward's turn of the same head has the sines' sign changed
    g, _, _, _ = rope.bwd(x, None, pos, torch.tensor(freq, dtype=torch.float64, device="cuda"), interleaved=interleaved)
    torch.cuda.synchronize()
    want = torch.tensor([[exact(p, f) for f in freq] for p in where], dtype=torch.float64)
    for out, sign in ((y, 1), (g, -1)):
        got = torch.stack((out[:, 0, first], out[:, 0, second]), -1).cpu().double()
        off = (got - want * torch.tensor([1.0, sign], dtype=torch.float64)).abs() / 2.0 ** -24
        assert float(off.max()) <= 4, (where[int(off.amax((1, 2)).argmax())], freq[int(off.amax((0, 2)).argmax())], float(off.max()))
