"""Group normalisation and its gradients against their float64 reference.

Tolerances.  Statistics, sums and values are fp32: a mean or a variance of m values, summed as a
tree of means, is off by at most about 2 log2(m) steps of 2^-24 (m <= 2^20: 40 * 2^-24 = 2.4e-6);
a result takes a difference with the mean and four more roundings.  1e-5 of the largest result
covers both, for inputs whose mean is not far larger than their spread (each test's inputs say by
how much it is, and its limit is that much larger).  A 16-bit result is off by half a step more.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import delta_ref
from tests.gpu_util import torch_dtype

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def sla():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2401_00912_amd import sla as S

    S.lib()
    return S


def close(got, ref, dtype, name, bar=1e-5):
    got = got.detach().double().cpu().numpy()
    real = ~np.isnan(ref)
    assert got.shape == ref.shape and np.isfinite(got[real]).all(), name
    if not real.any():
        return
    limit = HALF_STEP[dtype] * np.abs(ref[real]) + bar * max(np.abs(ref[real]).max(), 1e-30)
    limit += 2.0 ** -25 if dtype == "f16" else 0.0
    worst = np.max(np.abs(got[real] - ref[real]) / limit)
    assert worst <= 1.0, f"{name}: {worst:.3g} times its limit"


def check(S, lengths, C, G, dtype, act, behind=0, affine=True, seed=0, shift=0.5, bar=1e-5):
    import torch

    gen = torch.Generator().manual_seed(seed)
    n = behind + (lengths if isinstance(lengths, int) else int(sum(lengths)))
    dt = torch_dtype(dtype)
    x = (torch.randn(n, C, generator=gen) * (0.5 + torch.rand(C, generator=gen)) + shift).to(dt)
    dy = torch.randn(n, C, generator=gen).to(dt)
    w = 1 + 0.2 * torch.randn(C, generator=gen) if affine else None
    b = 0.2 * torch.randn(C, generator=gen) if affine else None
    offsets = None if isinstance(lengths, int) else np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    dev = lambda t: None if t is None else (torch.from_numpy(t) if isinstance(t, np.ndarray) else t).cuda()  # noqa: E731
    host = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    kw = dict(weight=dev(w), bias=dev(b), offsets=dev(offsets), activation=act)
    y, mean, rstd = S.forward_group_norm(dev(x), G, y=torch.full((n, C), 7.0, dtype=dt).cuda(), **kw)
    ry, rm, rr = delta_ref.group_norm_forward_ref(host(x), G, host(w), host(b), offsets, activation=act)
    close(mean, rm, "f32", "mean", bar)
    close(rstd, rr, "f32", "rstd", bar)
    close(y, ry, dtype, "y", bar)
    assert (y.float().cpu().numpy()[np.isnan(ry)] == 7.0).all(), "rows in no window are left as they were"
    dx, dw, db = S.backward_group_norm(dev(x), G, dev(dy), mean, rstd, dx=torch.full((n, C), 7.0, dtype=dt).cuda(), **kw)
    # relu's slope jumps where z = 0: the reference takes the kernel's own statistics, and z there is off
    # by 1e-6 of its size at most: rows where it is nearer to 0 than that are none in these inputs
    gx, gw, gb = delta_ref.group_norm_backward_ref(host(x), G, host(dy), mean.double().cpu().numpy(),
                                                   rstd.double().cpu().numpy(), host(w), host(b), offsets, act)
    close(dx, gx, dtype, "dx", bar)
    close(dw, gw, "f32", "dweight", bar)
    close(db, gb, "f32", "dbias", bar)
    assert (dx.float().cpu().numpy()[np.isnan(gx)] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("C,G", [(4, 1), (16, 4), (32, 1), (128, 8), (48, 4), (24, 2), (96, 3), (256, 32), (256, 1),
                                 (512, 2), (1024, 1), (2048, 16), (2048, 1), (1100, 5), (4096, 4), (4096, 1024),
                                 (3000, 6), (4000, 1)])
def test_rows(sla, C, G, dtype):
    check(sla, 37, C, G, dtype, "silu", seed=C + G)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("C,G", [(4, 1), (16, 4), (32, 1), (128, 8), (48, 4), (24, 2), (96, 3), (256, 32), (512, 2),
                                 (1024, 1), (2048, 16), (1100, 5), (4096, 4), (4000, 1)])
def test_short_windows(sla, C, G, dtype):
    check(sla, [5, 0, 1, 70, 33, 2, 0], C, G, dtype, "relu", behind=3, seed=C + G)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("C,G", [(4, 1), (16, 4), (32, 1), (128, 8), (48, 4), (24, 2), (256, 32), (512, 2), (1024, 1),
                                 (2048, 16), (1100, 5), (4096, 4)])
def test_long_windows(sla, C, G, dtype):
    check(sla, [700, 0, 1, 900], C, G, dtype, "silu", behind=5, seed=C + G)


@pytest.mark.parametrize("lengths", [1, 2, 3, 300, [1], [0], [0, 0], [1] * 50, [257], [16], [17], [40000], [20001, 1, 19999],
                                     [10000, 0, 0, 3]])
def test_lengths(sla, lengths):
    check(sla, lengths, 32, 4, "f32", "silu", seed=3)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("affine", [False, True])
def test_activations(sla, act, affine):
    for lengths in (64, [20, 44], [600, 424]):
        check(sla, lengths, 64, 8, "f32", act, affine=affine, seed=4)


@pytest.mark.parametrize("lengths", [64, [20, 44], [600, 3424]])
def test_mean_far_from_zero(sla, lengths):
    """A mean 1,000 times the spread: the variance is summed around it, so only the inputs' own steps
    and the mean's (2^-24 of it) count: 1,000 times the limit."""
    check(sla, lengths, 64, 8, "f32", "none", shift=1000.0, seed=5, bar=1e-2)


def test_no_rows(sla):
    import torch

    x = torch.empty(0, 64).cuda()
    y, mean, rstd = sla.forward_group_norm(x, 4)
    assert y.shape == (0, 64) and mean.shape == (0, 4)
    dx, dw, db = sla.backward_group_norm(x, 4, x, mean, rstd)
    assert (dw == 0).all() and (db == 0).all()


def test_not_finite_stays_in_its_group(sla):
    import torch

    for lengths in (40, [10, 30], [500, 600]):
        n = lengths if isinstance(lengths, int) else sum(lengths)
        off = None if isinstance(lengths, int) else torch.tensor(np.concatenate([[0], np.cumsum(lengths)]),
                                                                 dtype=torch.int32).cuda()
        x = torch.randn(n, 64, generator=torch.Generator().manual_seed(6)).cuda()
        clean = sla.forward_group_norm(x, 4, offsets=off)[0]
        x[5, 20] = torch.nan
        bad = sla.forward_group_norm(x, 4, offsets=off)[0]
        last = 6 if off is None else lengths[0]
        touched = torch.zeros(n, 64, dtype=torch.bool).cuda()
        touched[(5 if off is None else 0):last, 16:32] = True
        assert torch.equal(clean[~touched], bad[~touched]) and torch.isnan(bad[touched]).all()


def test_same_twice(sla):
    import torch

    x = torch.randn(5000, 128, generator=torch.Generator().manual_seed(7)).cuda().to(torch.bfloat16)
    off = torch.tensor([0, 2500, 2600, 5000], dtype=torch.int32).cuda()
    for o in (None, off):
        y, m, r = sla.forward_group_norm(x, 8, offsets=o, activation="silu")
        y2, m2, r2 = sla.forward_group_norm(x, 8, offsets=o, activation="silu")
        a, b = (sla.backward_group_norm(x, 8, y, m, r, offsets=o, activation="silu") for _ in range(2))
        assert torch.equal(y, y2) and torch.equal(m, m2) and torch.equal(r, r2)
        assert all(torch.equal(s, t) for s, t in zip(a, b))
