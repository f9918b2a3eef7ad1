"""The residual normalisation and its gradients against the float64 reference.

Tolerances.  A sum of at most 8,192 squares by 64 or 256 threads and a tree adds at most 32 + 14 roundings of
2^-24 to each term; a result takes two such statistics, their products and an activation, fewer than 120
roundings in all: 120 * 2^-24 = 7.2e-6, below 1e-5 of the largest result.  (The new residual rows and the
gradients are differences of terms of that size at most.)  A 16-bit result is off by half a step of its value
more.  A weight's gradient is a sum of up to 64 rows by one thread and 32 * 16 sums of threads, each a
rounding of what has been summed: 1e-5 of the sum of its terms' sizes.

The gradients of a norm are differences: rstd (d - hat mean(d hat)).  With one channel hat is 1 but for eps and
the difference is eps rstd^2 of its terms, 1e-5 and less of them, while each term is off by its own few
roundings whatever the difference is.  So dx and dresidual, and the sum that dpost_weight is of
them, are held to 1e-5 of the largest term and not of the largest difference."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import space_ref
from tests.gpu_util import torch_dtype
from tests.test_gpu_conv import close, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sla():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2401_00912_amd import sla as S

    S.lib()
    return S


num = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731


def check(S, n, C, dtype, rtype="same", act="silu", post=True, gate=True, weight=True, residual=True, more=True, scale=0.7,
          seed=0, eps=1e-5):
    import torch

    gen = torch.Generator().manual_seed(seed)
    dt = torch_dtype(dtype)
    rt = torch.float32 if rtype == "f32" else dt
    rname = "f32" if rtype == "f32" else dtype
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x, dy, g = (normal(n, C).to(dt).cuda() for _ in range(3))
    r, do = (normal(n, C).to(rt).cuda() for _ in range(2))
    w, pw = ((1 + 0.2 * normal(C)).cuda() for _ in range(2))
    r, g, w, pw, do = (t if on else None for t, on in ((r, residual), (g, gate), (w, weight), (pw, post), (do, more)))
    kw = dict(weight=w, post_weight=pw, gate=g, activation=act, scale=scale)
    rkw = dict(weight=num(w), post_weight=num(pw), gate=num(g), activation=act, scale=scale)
    y, ro, rstd, ps = S.forward_residual_norm(x, r, eps=eps, **kw)
    ry, rr, rs, rp = space_ref.rnorm_forward_ref(num(x), num(r), eps=eps, **rkw)
    if r is None:
        rname = dtype
    close(y, ry, dtype, "y")
    close(ro, rr, rname, "residual_out")
    assert np.abs(num(rstd) / rs - 1).max() < 1e-5
    assert (ps is None) == (not post) and (ps is None or np.abs(num(ps) / rp - 1).max() < 1e-5)
    do = None if do is None else do.to(ro.dtype)
    got = S.backward_residual_norm(x, ro, dy, rstd, post_rstd=ps, dresidual_out=do, **kw)
    ref = space_ref.rnorm_backward_ref(num(x), num(ro), num(dy), num(rstd), post_rstd=num(ps), dresidual_out=num(do), **rkw)
    dx, dr, dw, dpw, dg = got
    terms = np.abs(num(rstd)[:, None] * num(dy) * (1 if w is None else num(w)))
    terms = terms.max(-1, keepdims=True) + (0 if do is None else np.abs(num(do)).max(-1, keepdims=True))
    close(dr, ref[1], rname, "dresidual", size=terms.max())
    d = scale * terms * (1 if g is None else np.abs(space_ref._act(act, num(g))).max(-1, keepdims=True))
    close(dx, ref[0], dtype, "dx", size=(d if not post else d * num(ps)[:, None] * np.abs(num(pw)).max()).max())
    hat = np.abs(num(ro) * num(rstd)[:, None])
    assert (dw is None) == (not weight) and (dpw is None) == (not post) and (dg is None) == (not gate)
    if weight:
        within(dw, ref[2], 1e-5 * (np.abs(num(dy)) * hat).sum(0), "dweight")
    if gate:
        u = num(x) if not post else num(x) * num(ps)[:, None] * num(pw)
        close(dg, ref[4], dtype, "dgate", size=(scale * terms * 1.1 * np.abs(u).max(-1, keepdims=True)).max())
    if post:
        d = scale * terms * (1 if g is None else np.abs(space_ref._act(act, num(g))))
        within(dpw, ref[3], 1e-5 * 2 * (d * np.abs(num(x)) * num(ps)[:, None]).sum(0), "dpost_weight")


@pytest.mark.parametrize("dtype,rtype", [("f32", "same"), ("f16", "same"), ("f16", "f32"), ("bf16", "same"), ("bf16", "f32")])
@pytest.mark.parametrize("C", [1, 3, 8, 64, 130, 256, 500, 512, 1000, 1024, 2048, 2050, 4096, 5000, 8192, 8191])
def test_widths(sla, C, dtype, rtype):
    check(sla, 11, C, dtype, rtype, seed=C)


@pytest.mark.parametrize("n", [0, 1, 2, 3, 4, 5, 63, 513, 2049, 9000])
def test_rows(sla, n):
    if n:
        for C in (96, 1280):
            check(sla, n, C, "f32", seed=n)
            check(sla, n, C, "bf16", "f32", seed=n)
    else:
        import torch

        x = torch.zeros(0, 96).cuda()
        w = torch.ones(96).cuda()
        y, ro, rstd, _ = sla.forward_residual_norm(x, x, weight=w)
        assert y.shape == x.shape and rstd.shape == (0,)
        _, _, dw, _, _ = sla.backward_residual_norm(x, ro, x, rstd, weight=w)
        assert (dw == 0).all()


@pytest.mark.parametrize("kw", [dict(post=False), dict(gate=False), dict(weight=False), dict(residual=False), dict(more=False),
                                dict(act="none"), dict(act="relu"), dict(scale=1.0), dict(eps=0.0),
                                dict(post=False, gate=False), dict(post=False, gate=False, weight=False, residual=False)])
def test_options(sla, kw):
    for C in (200, 2048, 77):
        check(sla, 20, C, "f32", seed=1, **kw)
        check(sla, 20, C, "bf16", "f32", seed=2, **kw)


def test_in_place(sla):
    import torch

    gen = torch.Generator().manual_seed(3)
    x, g, dy, r, do = (torch.randn(300, 1024, generator=gen).cuda() for _ in range(5))
    pw = torch.rand(1024, generator=gen).cuda()
    y, ro, rstd, ps = sla.forward_residual_norm(x, r, post_weight=pw, gate=g)
    mine = r.clone()
    y2, _, _, _ = sla.forward_residual_norm(x, mine, post_weight=pw, gate=g, residual_out=mine)
    assert torch.equal(y, y2) and torch.equal(mine, ro)
    kw = dict(post_weight=pw, post_rstd=ps, gate=g)
    want = sla.backward_residual_norm(x, ro, dy, rstd, dresidual_out=do, **kw)
    mine = do.clone()
    got = sla.backward_residual_norm(x, ro, dy, rstd, dresidual_out=mine, dresidual=mine, **kw)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, want))


def test_values_whose_squares_leave_the_range(sla):
    """Rows of 1e30 and of 1e-30 are normalised like others; zeros and infinities stay in their rows."""
    import torch

    for C in (64, 2048, 100):
        gen = torch.Generator().manual_seed(C)
        x, r = (torch.randn(6, C, generator=gen).cuda() for _ in range(2))
        size = torch.tensor([1.0, 1e30, 1e-30, 0.0, 1.0, 1e-20]).cuda()[:, None]
        x, r = x * size, r * size
        x[4, 5] = float("inf")
        pw = torch.rand(C, generator=gen).cuda()
        y, ro, rstd, ps = sla.forward_residual_norm(x, r, post_weight=pw, eps=1e-38, scale=1.0)
        rows = [0, 1, 2, 3, 5]
        ry, rr, rs, rp = space_ref.rnorm_forward_ref(num(x[rows]), num(r[rows]), post_weight=num(pw), eps=1e-38)
        for i, k in enumerate(rows):
            # eps itself is a denormal step off: 2^-149 of 1e-38
            close(y[k:k + 1], ry[i:i + 1], "f32", f"y of row {k}")
            close(ro[k:k + 1], rr[i:i + 1], "f32", f"residual of row {k}")
        assert not torch.isfinite(y[4]).all() and torch.isfinite(y[[0, 1, 2, 3, 5]]).all()


@pytest.mark.parametrize("eps", [1e-5, 1e-12, 1e-21, 1e-30, 1000.0])
def test_small_rows_beside_any_eps(sla, eps):
    """Rows whose squares are far below eps are scaled by 1 / sqrt(eps); those far above are normalised."""
    import torch

    for C in (64, 2048, 100):
        gen = torch.Generator().manual_seed(C)
        size = torch.tensor([1.0, 1e-8, 1e-13, 1e-16, 1e-25, 1e-30, 1e-38, 0.0]).cuda()[:, None]
        r = torch.randn(8, C, generator=gen).cuda() * size
        zero = torch.zeros_like(r)
        y, _, rstd, _ = sla.forward_residual_norm(zero, r, eps=eps)
        ry, _, rs, _ = space_ref.rnorm_forward_ref(num(zero), num(r), eps=np.float64(np.float32(eps)))
        # a statistic is off by its sum's roundings; a denormal input by 2^-149
        assert (np.abs(num(rstd) / rs - 1) < 1e-5).all()
        for k in range(8):
            close(y[k:k + 1], ry[k:k + 1], "f32", f"row {k}", size=1e-38 * rs[k])


def test_parameters_at_any_address(sla):
    import torch

    gen = torch.Generator().manual_seed(5)
    x, r, g, dy = (torch.randn(9, 512, generator=gen).cuda() for _ in range(4))
    w, pw = (torch.randn(512, generator=gen).cuda() for _ in range(2))
    odd = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    kw = dict(weight=w, post_weight=pw, gate=g, activation="silu")
    a = sla.forward_residual_norm(x, r, **kw)
    want = sla.backward_residual_norm(x, a[1], dy, a[2], post_rstd=a[3], **kw)
    kw.update(weight=odd(w), post_weight=odd(pw))
    b = sla.forward_residual_norm(x, r, **kw)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    got = sla.backward_residual_norm(x, a[1], dy, a[2], post_rstd=a[3], **kw)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    # rows there too: one value a load, another order of sums
    kw.update(gate=odd(g))
    c = sla.forward_residual_norm(odd(x), odd(r), **kw)
    got = sla.backward_residual_norm(odd(x), odd(a[1]), odd(dy), a[2], post_rstd=a[3], **kw)
    for p, q in zip((*a, *want), (*c, *got)):
        assert (p - q).abs().max() <= 2e-5 * p.abs().max()


def test_gradients_by_differences(sla):
    import torch

    gen = torch.Generator().manual_seed(4)
    n, C = 9, 60
    r = {k: torch.randn(n, C, generator=gen).cuda() for k in ("x", "residual", "gate")}
    r.update(weight=torch.rand(C, generator=gen).cuda() + 0.5, post_weight=torch.rand(C, generator=gen).cuda() + 0.5)
    dy, do = (torch.randn(n, C, generator=gen).cuda() for _ in range(2))
    kw = dict(weight=r["weight"], post_weight=r["post_weight"], gate=r["gate"], activation="silu", scale=0.5)
    _, ro, rstd, ps = sla.forward_residual_norm(r["x"], r["residual"], **kw)
    got = dict(zip(("x", "residual", "weight", "post_weight", "gate"),
                   sla.backward_residual_norm(r["x"], ro, dy, rstd, post_rstd=ps, dresidual_out=do, **kw)))

    def loss(r):
        h = {k: num(v) for k, v in r.items()}
        y, o, _, _ = space_ref.rnorm_forward_ref(h["x"], h["residual"], h["weight"], h["post_weight"], h["gate"], "silu", 0.5)
        return (y * num(dy)).sum() + (o * num(do)).sum()

    for name, grad in got.items():
        d = torch.randn(r[name].shape, generator=gen, dtype=torch.float64)
        up, down = (loss({**r, name: r[name].double().cpu() + s * 1e-4 * d}) for s in (1, -1))
        mine = float((grad.double().cpu() * d).sum())
        assert abs((up - down) / 2e-4 - mine) <= 1e-5 * float(grad.double().norm() * d.norm()), name
