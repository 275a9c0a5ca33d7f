"""Sine and cosine of the paged calls' rotation: what comes out for (1, 0) and (0, 1), against 64 bits."""
import math

import pytest
import torch

from paper_2510_25600_b200 import binding as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_sine_and_cosine(interleaved):
    """sincospif is off by one unit in the last place at most, 2^-24 for results up to 1; the part of the turn that 32 bits do not hold is
    added with one more rounding, 2^-25 (its own errors, and the square of it, are below 2^-44); products with 1 and 0 and their sum are exact."""
    n, d = 4096, 128
    g = torch.Generator().manual_seed(70)
    pos = torch.cat([torch.arange(1024), torch.randint(0, 1 << 20, (n - 1024,), generator=g)]).to(torch.int32)
    freq = 1000000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
    angle = pos.double()[:, None] * freq
    a, b = (slice(0, d, 2), slice(1, d, 2)) if interleaved else (slice(0, d // 2), slice(d // 2, d))
    worst = 0.0
    for first in (True, False):
        q = torch.zeros((n, 1, d))
        q[..., a if first else b] = 1
        out = P.purekv_append_paged(None, None, None, None, None, None, q=q.cuda(), positions=pos.cuda(), inv_freq=freq.cuda(), interleaved=interleaved).cpu().double()[:, 0]
        want = (torch.cos(angle), torch.sin(angle)) if first else (-torch.sin(angle), torch.cos(angle))
        worst = max(worst, *(float((out[:, s] - w).abs().max()) for s, w in zip((a, b), want)))
    assert worst <= 1.5 * 2.0 ** -24 + 2.0 ** -44 + math.ulp(float(angle.max())), worst * 2.0 ** 24
