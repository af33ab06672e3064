"""Angles of far rotary positions against 90 decimal digits: what is left is the rounding of a fraction of a turn to fp32, and of its sine and cosine."""
import math
import random
from decimal import Decimal, localcontext

import pytest
import torch

pytestmark = pytest.mark.gpu


def turns(positions, freqs):
    """positions * freqs / (2 pi), less whole turns, rounded to 64 bits."""
    with localcontext() as c:
        c.prec = 90

        def arctan_of_inverse(n):
            t = s = Decimal(1) / n
            k = 1
            while abs(t) > Decimal(10) ** -85:
                t, k = t / -(n * n), k + 2
                s += t / k
            return s

        two_pi = 8 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239))         # Machin
        rows = []
        for p in positions:
            t = [Decimal(p) * Decimal(f) / two_pi for f in freqs]
            rows.append([float(x - x.to_integral_value()) for x in t])
    return torch.tensor(rows, dtype=torch.float64)


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_angles_are_off_by_their_rounding(inverse, interleaved):
    from paper_2405_18428_b200 import dig
    rng = random.Random(4)
    freqs, axes = dig.dig_rope_freqs((8,))
    pos = [0, 1, 2 ** 31 - 1, -2 ** 31] + [rng.randrange(2 ** 30, 2 ** 31) * rng.choice((1, -1)) for _ in range(3000)] + [rng.randrange(2 ** 20) for _ in range(500)]
    q = torch.zeros(1, len(pos), 1, 16, device="cuda")
    q[..., 0::2 if interleaved else 1] = 1
    if not interleaved:
        q[..., 8:] = 0
    out, _ = dig.dig_rope(q, None, torch.tensor(pos, dtype=torch.int32, device="cuda")[:, None].contiguous(), freqs, axes, interleaved=interleaved, inverse=inverse)
    out = out[0, :, 0].double().cpu()
    cos, sin = (out[:, 0::2], out[:, 1::2]) if interleaved else (out[:, :8], out[:, 8:])
    angle = 2 * math.pi * turns(pos, freqs) * (-1 if inverse else 1)
    # half a step of a fraction of half a turn below 1 is 2^-25, times pi; sine and cosine two units in the last place below 1, 2^-24 each; the
    # turns by 1 and 0 are exact
    lim = math.pi * 2.0 ** -25 + 2 * 2.0 ** -24
    assert (cos - angle.cos()).abs().max() <= lim and (sin - angle.sin()).abs().max() <= lim


def test_angles_of_any_finite_frequency_are_finite():
    from paper_2405_18428_b200 import dig
    pos = torch.tensor([[2 ** 31 - 1], [-2 ** 31], [0], [7]], dtype=torch.int32, device="cuda")
    q = torch.ones(1, 4, 1, 16, device="cuda")
    out, _ = dig.dig_rope(q, None, pos, [1e30, -1e30, 1e-30, 1e15, 0.0, 5e-324, 3.0, -3.0], [0] * 8)
    assert torch.isfinite(out).all() and out.abs().max() <= 1.5
    assert (out[0, 2] == 1).all()                    # position 0 turns nothing
