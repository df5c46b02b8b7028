"""The rotation's angle at far positions, against arithmetic of 60 digits."""
import math
from decimal import Decimal, localcontext

import pytest
import torch

pytestmark = pytest.mark.gpu

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def _turned(pos, freq):
    """cosine and sine of pos * freq, the whole turns taken out exactly."""
    with localcontext() as c:
        c.prec = 60
        turns = Decimal(pos) * Decimal(freq) / (2 * PI)
        rest = float((turns - turns.to_integral_value()) * 2 * PI)
    return math.cos(rest), math.sin(rest)


@pytest.mark.parametrize("low,high", [(0, 1 << 12), (1 << 26, 1 << 27), (1 << 30, 2 ** 31 - 1), (-2 ** 31, -1 << 30)])
def test_angles_lose_nothing_far_out(low, high):
    from paper_2512_21571_b200 import binding as nnc
    g = torch.Generator().manual_seed(high & 0xffff)
    pos = torch.randint(low, high, (48,), generator=g)
    freq = torch.cat([torch.rand(28, generator=g, dtype=torch.float64) * 1.5 + 0.5, nnc.rope_frequencies(128, 1e6, device="cpu")[0][::16]])
    half = freq.numel()
    x = torch.zeros(len(pos), 1, 2 * half, device="cuda")
    x[..., :half] = 1.0                                                  # pairs (1, 0) become (cos, sin)
    y = nnc.op_rope(x, pos.int().cuda(), freq.cuda()).double().cpu()
    want = [[_turned(int(p), f) for f in freq.tolist()] for p in pos]
    want = torch.tensor([[a[0] for a in row] + [a[1] for a in row] for row in want], dtype=torch.float64)
    # the angle: 2^-28 turns, so 2^-25.3; cosine and sine of it: one unit of a value up to 1, 2^-24; the products are exact
    assert ((y[:, 0] - want).abs() <= 2.0 ** -25.3 + 2.0 ** -24).all(), (y[:, 0] - want).abs().max().item() * 2 ** 24
