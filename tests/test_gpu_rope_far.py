"""Rotary positions at the farthest positions, against angles in 70 digits."""
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

import paper_2605_11478_amd as fq

pytestmark = pytest.mark.gpu

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628621")


def turns(positions, freqs):
    """cos and sin of positions x freqs (float64): the angle less whole turns, exactly."""
    with localcontext() as c:
        c.prec = 70
        a = np.array([[float((Decimal(int(p)) * Decimal(float(f))).remainder_near(2 * PI)) for f in freqs]
                      for p in positions])
    return np.cos(a), np.sin(a)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_angles(device, layout):
    """A pair (1, 0) becomes (cos, sin), each off by 2^-23 at most: its argument, an eighth of a
    turn rounded to float (2^-25 of it), and its own rounding."""
    rng = np.random.default_rng(6)
    half = 128
    freqs = np.concatenate([rng.uniform(0.5, 1.0, half - 8), [1.0, 0.1, 3.0, 7.7, 0.5, 1e-4, 1e-9, 0.9999999]])
    positions = np.concatenate([rng.integers(2 ** 30, 2 ** 31, 30), [2 ** 31 - 1, -2 ** 31, 2 ** 28 + 1, 1, 0, -7]])
    x = torch.zeros(len(positions), 1, 2 * half, device=device)
    first, second = ((slice(0, half), slice(half, None)) if layout == "half"
                     else (slice(0, None, 2), slice(1, None, 2)))
    x[..., first] = 1
    y, _ = fq.rope(x, None, torch.from_numpy(positions.astype(np.int32)).to(device),
                   torch.from_numpy(freqs).to(device), layout)
    got = y[:, 0].cpu().double().numpy()
    c, s = turns(positions, freqs)
    assert np.abs(got[:, first] - c).max() <= 2.0 ** -23 and np.abs(got[:, second] - s).max() <= 2.0 ** -23
