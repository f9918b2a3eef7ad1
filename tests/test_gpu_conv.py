"""The short causal convolution, its gradients and its single rows against the float64 reference.

Tolerances.  A sum of at most 8 products and a bias takes 9 roundings of 2^-24 of the sum of their sizes,
the activation and its slope a few more: 16 * 2^-24 = 9.6e-7 of that sum of sizes (dx: of 8 such products
of gradients), below 1e-5 of the largest result as long as the sums do not cancel to less than a tenth of
their terms in every row; a 16-bit result is off by half a step of its value more.  The weights' gradients
are fp32 sums of up to 256 rows by one thread, then of the threads' sums: each of at most 256 + 64
roundings is 2^-24 of what has been summed, so 320 * 2^-24 = 1.9e-5 of the sum of the terms' sizes
bounds them, with 1e-6 for the terms themselves."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import space_ref
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


def close(got, ref, dtype, name, bar=1e-5, size=None):
    """Every value within half a step of its type and `bar` of the largest (or of `size`, the largest term of
    results that cancel); NaN where the reference has it stands for a row that is left as it was (7)."""
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, name
    real = ~np.isnan(ref)
    assert (got[~real] == 7.0).all(), f"{name}: rows in no window are left as they were"
    got, ref = got[real], ref[real]
    if not ref.size:
        return
    assert np.isfinite(got).all(), name
    limit = HALF_STEP[dtype] * np.abs(ref) + bar * max(np.abs(ref).max(), size or 1e-30) + (2.0 ** -25 if dtype == "f16" else 0)
    worst = np.max(np.abs(got - ref) / limit)
    assert worst <= 1.0, f"{name}: {worst:.3g} times its limit"


def within(got, ref, limit, name):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    worst = np.max(np.abs(got - ref) / np.maximum(limit, 1e-30))
    assert worst <= 1.0, f"{name}: {worst:.3g} times its limit"


class Case:
    def __init__(self, lengths, C, K, dtype, act="silu", seed=0, bias=True, state=False, grads=True, order=False,
                 front=0, behind=0, strided=False):
        import torch

        gen = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        self.n, self.w, self.act, self.dtype = front + sum(lengths) + behind, len(lengths), act, dtype
        n, dt = self.n, torch_dtype(dtype)
        self.offsets = (front + np.concatenate([[0], np.cumsum(lengths)])).astype(np.int32)
        wide = normal(n, 3 * C + 5).to(dt).cuda()
        self.x = wide[:, C + 2:2 * C + 2] if strided else wide[:, :C].contiguous()
        self.dy = wide[:, 2 * C + 3:3 * C + 3] if strided else normal(n, C).to(dt).cuda()
        self.weight = (normal(C, K) / K ** 0.5).cuda()
        self.bias = (0.5 * normal(C)).cuda() if bias else None
        self.state = normal(self.w, K - 1, C).to(dt).cuda() if state else None
        self.dstate = normal(self.w, K - 1, C).to(dt).cuda() if state else None
        self.order = torch.randperm(n, generator=gen).to(torch.int32).cuda() if order else None
        self.off = torch.from_numpy(self.offsets).cuda()
        self.new = lambda: torch.full((n, C), 7.0, dtype=dt).cuda()
        self.kw = dict(bias=self.bias, activation=act, order=self.order, state=self.state)
        self.host = {k: None if v is None else v.double().cpu().numpy()
                     for k, v in dict(x=self.x, dy=self.dy, w=self.weight, b=self.bias, s=self.state, d=self.dstate).items()}
        self.ref_kw = dict(bias=self.host["b"], activation=act, state=self.host["s"],
                           order=None if self.order is None else self.order.cpu().numpy())

    def check(self, S):
        h = self.host
        y, st = S.forward_short_conv(self.x, self.weight, self.off, y=self.new(), **self.kw)
        ry, rs = space_ref.conv_forward_ref(h["x"], h["w"], self.offsets, **self.ref_kw)
        close(y, ry, self.dtype, "y")
        assert (st.double().cpu().numpy() == rs).all(), "states are inputs, exactly"
        dx, dw, db, ds = S.backward_short_conv(self.x, self.weight, self.off, self.dy, dstate=self.dstate, dx=self.new(),
                                               **self.kw)
        gx, gw, gb, gs = space_ref.conv_backward_ref(h["x"], h["w"], self.offsets, h["dy"], dstate=h["d"], **self.ref_kw)
        close(dx, gx, self.dtype, "dx")
        if self.state is not None:
            close(ds, gs, self.dtype, "dstate_in")
        # |dz| <= 1.1 |dy|, so the terms' sizes are at most those of |dy| and |x|
        if h["s"] is not None:
            h = {**h, "s": np.abs(h["s"])}
        _, sw, sb, _ = space_ref.conv_backward_ref(np.abs(h["x"]), np.zeros_like(h["w"]), self.offsets, np.abs(h["dy"]),
                                                   activation="none", state=h["s"], order=self.ref_kw["order"])
        within(dw, gw, 1.1 * 2.0e-5 * sw, "dweight")
        if self.bias is not None:
            within(db, gb, 1.1 * 2.0e-5 * sb, "dbias")
        else:
            assert db is None
        return y, st, dx, dw, db, ds


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("C", [1, 3, 8, 12, 40, 130, 520])
def test_widths(sla, dtype, K, C):
    Case([5, 0, 1, 70, 33, 2, 0, 3], C, K, dtype, seed=C + K, state=K % 2 == 0, front=2, behind=3).check(sla)


@pytest.mark.parametrize("lengths", [[1], [0], [2], [3], [7, 8, 9], [16], [17], [15, 1, 16, 0, 0, 33], [1] * 50, [300],
                                     [0, 0, 1], [2] * 9, [1000, 3]])
def test_lengths(sla, lengths):
    for state in (False, True):
        Case(lengths, 24, 4, "f32", seed=3, state=state).check(sla)
        Case(lengths, 9, 8, "bf16", seed=4, state=state, behind=1).check(sla)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("bias", [False, True])
def test_activations(sla, act, bias):
    Case([40, 90, 3], 64, 4, "f32", act, seed=5, bias=bias, state=True).check(sla)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 64, 2048])
def test_strided_rows_and_order(sla, dtype, C):
    Case([30, 4, 50], C, 4, dtype, seed=6, strided=True, state=True, behind=2).check(sla)
    Case([30, 4, 50], C, 4, dtype, seed=7, order=True, state=True, behind=2, front=1).check(sla)
    Case([30, 4, 50], C, 3, dtype, seed=8, order=True, strided=True).check(sla)


def test_long_and_wide(sla):
    """Strips of several batches of rows, several workgroups across the channels."""
    Case([5000, 0, 2777], 4096, 4, "bf16", seed=9, state=True).check(sla)
    Case([30000], 72, 4, "f32", seed=10).check(sla)


def test_aligned_rows_are_the_odd_ones(sla):
    """The same values by 16 bytes and one by one: equal bits."""
    import torch

    for dtype in ("f32", "f16", "bf16"):
        c = Case([100, 7, 64], 64, 4, dtype, seed=11, state=True)
        a = c.check(sla)
        buf = torch.zeros(c.n, 67, dtype=c.x.dtype, device="cuda")
        buf[:, 1:65] = c.x
        y, st = sla.forward_short_conv(buf[:, 1:65], c.weight, c.off, y=c.new(), **c.kw)
        g = sla.backward_short_conv(buf[:, 1:65], c.weight, c.off, c.dy, dstate=c.dstate, dx=c.new(), **c.kw)
        for p, q in zip(a, (y, st, *g)):
            assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("C,K", [(1, 2), (7, 4), (64, 4), (2056, 3), (4096, 8), (300, 5)])
def test_single_rows(sla, dtype, C, K):
    import torch

    gen = torch.Generator().manual_seed(C)
    dt = torch_dtype(dtype)
    slots = torch.tensor([3, 0, 3, -1, 5, 3, 7, 0], dtype=torch.int32)
    wide = torch.randn(8, 2 * C, generator=gen).to(dt).cuda()
    w, b = (torch.randn(C, K, generator=gen) / K ** 0.5).cuda(), torch.randn(C, generator=gen).cuda()
    for x in (wide[:, :C], wide[:, C:].contiguous()):
        pool = torch.randn(7, K - 1, C, generator=gen).to(dt).cuda()
        num = lambda t: t.double().cpu().numpy()  # noqa: E731
        ry, rs = space_ref.conv_step_ref(num(pool), slots.numpy(), num(x), num(w), num(b), "silu")
        y = sla.step_short_conv(pool, slots.cuda(), x, w, b, "silu", y=torch.full((8, C), 7.0, dtype=dt).cuda())
        close(y, ry, dtype, "y")
        assert (num(pool) == rs).all()


def test_steps_are_the_forward(sla):
    """Row by row over a pool gives the bits that all rows at once give."""
    import torch

    c = Case([37], 136, 4, "bf16", seed=12, state=True)
    y, st = sla.forward_short_conv(c.x, c.weight, c.off, **c.kw)
    pool, slot = c.state.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    got = [sla.step_short_conv(pool, slot, c.x[t:t + 1], c.weight, c.bias, "silu") for t in range(37)]
    assert torch.equal(torch.cat(got), y) and torch.equal(pool, st)
    # and a sequence cut in two
    a, s1 = sla.forward_short_conv(c.x[:20], c.weight, torch.tensor([0, 20], dtype=torch.int32).cuda(), **c.kw)
    b, s2 = sla.forward_short_conv(c.x[20:], c.weight, torch.tensor([0, 17], dtype=torch.int32).cuda(),
                                   **{**c.kw, "state": s1})
    assert torch.equal(torch.cat([a, b]), y) and torch.equal(s2, st)


def test_values_that_are_not_finite_stay_in_their_rows(sla):
    import torch

    c = Case([20, 20], 8, 4, "f32", seed=13, state=True)
    c.x[5, 3], c.x[19, 2] = float("nan"), float("inf")
    y, st = sla.forward_short_conv(c.x, c.weight, c.off, **c.kw)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[5:9, 3] = True
    want[19, 2] = bad[19, 2]   # infinity or silu's 0
    assert torch.equal(bad, want)
    assert not torch.isfinite(st[0]).all() and torch.isfinite(st[1]).all()


def test_gradients_by_differences(sla):
    import torch

    c = Case([40, 3, 21], 16, 4, "f32", seed=14, state=True)
    dx, dw, db, ds = sla.backward_short_conv(c.x, c.weight, c.off, c.dy, dstate=c.dstate, **c.kw)
    rows = dict(x=c.x, w=c.weight, b=c.bias, s=c.state)

    def loss(r):
        host = {k: v.double().cpu().numpy() for k, v in r.items()}
        y, st = space_ref.conv_forward_ref(host["x"], host["w"], c.offsets, host["b"], "silu", state=host["s"])
        return (y * c.host["dy"]).sum() + (st * c.host["d"]).sum()

    gen = torch.Generator().manual_seed(1)
    for name, grad in zip(("x", "w", "b", "s"), (dx, dw, db, ds)):
        d = torch.randn(rows[name].shape, generator=gen, dtype=torch.float64)
        up, down = (loss({**rows, name: rows[name].double().cpu() + s * 1e-4 * d}) for s in (1, -1))
        got = float((grad.double().cpu() * d).sum())
        # the difference's own error is 1e-8 of a third derivative; the gradient's 1e-5 of its size
        assert abs((up - down) / 2e-4 - got) <= 1e-5 * float(grad.double().norm() * d.norm()), name


WRONG = ([0, 200, 100, 300, 250, 700], [-5, 300, 900, 10, 10, 2000], [700, 600, 500, 400, 0, 700], [0, 2000, 0, 2000, 0, 2000])


@pytest.mark.parametrize("offsets", WRONG)
def test_wrong_offsets_stay_in_range(sla, offsets):
    """Offsets out of order or range, an order past both ends: nothing outside the outputs is written."""
    import torch

    n, C, K = 700, 24, 4
    c = Case([n], C, K, "bf16", seed=15)
    off = torch.tensor(offsets, dtype=torch.int32).cuda()
    w = len(offsets) - 1
    state = torch.randn(w, K - 1, C).to(c.x.dtype).cuda()
    bad = torch.arange(n, dtype=torch.int32).cuda() * 3 - n
    for order in (None, bad):
        y = torch.full((3, n, C), 7.0, dtype=c.x.dtype).cuda()
        dx, fin = y.clone(), torch.full((3, w, K - 1, C), 7.0, dtype=c.x.dtype).cuda()
        kw = dict(bias=c.bias, activation="silu", order=order, state=state)
        sla.forward_short_conv(c.x, c.weight, off, y=y[1], final_state=fin[1], **kw)
        sla.backward_short_conv(c.x, c.weight, off, c.dy, dstate=state, dx=dx[1], **kw)
        torch.cuda.synchronize()
        for t in (y, dx, fin):
            assert (t[0] == 7.0).all() and (t[2] == 7.0).all()
