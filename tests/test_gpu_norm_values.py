"""Group normalisation at the ends of its activations."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sla():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2401_00912_amd import sla as S

    S.lib()
    return S


@pytest.mark.parametrize("lengths", [24, [10, 14], [400, 300]])
def test_silu_far_from_zero(sla, lengths):
    """silu and its slope where z is a bias of any size: 0 and 0 far below zero (infinitely far too), z and 1 far
    above it.  x is constant, so z is the bias itself; y is rounded once, and 1.6e-38 * 87, the sigmoid's end at
    -87, is all that it may be off below zero."""
    import torch

    n = lengths if isinstance(lengths, int) else sum(lengths)
    off = None if isinstance(lengths, int) else torch.tensor(np.concatenate([[0], np.cumsum(lengths)]),
                                                             dtype=torch.int32).cuda()
    bias = torch.tensor([-torch.inf, -3e38, -1e38, -1e30, -1000.0, -88.0, -86.0, -1.0, 0.0, 1.0, 86.0, 88.0, 1000.0, 1e30,
                         3e38, torch.inf]).cuda()
    x = torch.ones(n, 16).cuda()
    y, mean, rstd = sla.forward_group_norm(x, 1, weight=torch.ones(16).cuda(), bias=bias, offsets=off, activation="silu")
    z = bias.double().cpu().numpy()
    inner = np.abs(z) < 500
    zi = z[inner]
    want, slope = np.where(z > 0, z, 0.0), (z > 0).astype(float)
    want[inner] = zi / (1 + np.exp(-zi))
    s = 1 / (1 + np.exp(-zi))
    slope[inner] = s * (1 + zi * (1 - s))
    got = y.double().cpu().numpy()
    end = np.isinf(want)
    assert (got[:, end] == np.inf).all()
    assert (np.abs(got[:, ~end] - want[~end]) <= 1e-6 * np.abs(want[~end]) + 1.5e-36).all()
    # weight 0: dx is 0, and dbias the sum of dy times the slope
    dy = torch.ones(n, 16).cuda()
    dx, dw, db = sla.backward_group_norm(x, 1, dy, mean, rstd, weight=torch.zeros(16).cuda(), bias=bias, offsets=off,
                                         activation="silu")
    assert (np.abs(db.double().cpu().numpy() - n * slope) <= 1e-6 * n * np.abs(slope) + n * 1.5e-36).all()
    assert (dx == 0).all() and torch.isfinite(dw).all()
