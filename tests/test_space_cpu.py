"""CPU tests of the short convolution, the selective scan and the residual normalisation: what the entry
points and the binding refuse (all of it before anything is launched), and their float64 references
against other forms of the same operators."""
from __future__ import annotations

import os

import numpy as np
import pytest

from oracle import space_ref
from paper_2401_00912_amd import sla

FAKE = 1 << 20  # a 256-aligned fake device address: never dereferenced, every call below fails validation
BIG = 1 << 40   # workspace bytes that are enough for every size here


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sla.LIB_PATH):
        from paper_2401_00912_amd import build

        build.build()
    return sla.lib()


def call(f, order, defaults, kw):
    a = dict(defaults)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return f(*(a[x] for x in order))


def code(name):
    return getattr(sla, "SLA_E_" + name)


# addresses that differ, so that no output is an input
names = iter(range(1, 100))
at = lambda: FAKE * (1 + next(names))  # noqa: E731

CONV = dict(offsets=at(), n=100, W=3, order=None, dtype=1, C=64, K=4, act=2, x=at(), ldx=128, w=at(), b=at(), s=None,
            y=at(), so=None, dy=at(), lddy=64, ds=None, dx=at(), dw=at(), db=at(), dsi=None, ws=at(), nbytes=BIG, stream=None,
            slots=at(), pool=at())
CONV_FWD = ["offsets", "n", "W", "order", "dtype", "C", "K", "act", "x", "ldx", "w", "b", "s", "y", "so", "stream"]
CONV_BWD = ["offsets", "n", "W", "order", "dtype", "C", "K", "act", "x", "ldx", "w", "b", "s", "dy", "lddy", "ds", "dx", "dw",
            "db", "dsi", "ws", "nbytes", "stream"]
CONV_STEP = ["slots", "n", "W", "dtype", "C", "K", "act", "pool", "x", "ldx", "w", "b", "y", "stream"]


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), "ARG"), (dict(n=2 ** 31 - 1), "ARG"), (dict(W=0), "ARG"), (dict(dtype=3), "ARG"), (dict(dtype=-1), "ARG"),
    (dict(C=0), "ARG"), (dict(C=65537, ldx=1 << 20), "UNSUPPORTED"), (dict(K=1), "UNSUPPORTED"), (dict(K=9), "UNSUPPORTED"),
    (dict(W=2 ** 23), "UNSUPPORTED"), (dict(n=2 ** 31 - 2), "UNSUPPORTED"), (dict(act=3), "ARG"), (dict(act=-1), "ARG"),
    (dict(x=None), "ARG"), (dict(x=FAKE + 1), "ARG"), (dict(ldx=63), "ARG"), (dict(w=None), "ARG"), (dict(w=FAKE + 2), "ARG"),
    (dict(b=FAKE + 2), "ARG")])
def test_conv_refusals(L, kw, want):
    for f, order in ((L.sla_forward_short_conv, CONV_FWD), (L.sla_backward_short_conv, CONV_BWD),
                     (L.sla_step_short_conv, CONV_STEP)):
        assert call(f, order, CONV, kw) == code(want)


def test_conv_refusals_of_one(L):
    f = L.sla_forward_short_conv
    for kw in (dict(offsets=None), dict(offsets=FAKE + 2), dict(order=FAKE + 1), dict(y=None), dict(y=FAKE + 1),
               dict(y=CONV["x"]), dict(s=FAKE + 1), dict(so=FAKE + 1), dict(s=FAKE, so=FAKE)):
        assert call(f, CONV_FWD, CONV, kw) == sla.SLA_E_ARG, kw
    assert call(f, CONV_FWD, CONV, dict(n=0, x=None, y=None)) == sla.SLA_OK
    f = L.sla_backward_short_conv
    for kw in (dict(dy=None), dict(lddy=63), dict(dx=None), dict(dw=None), dict(db=FAKE + 1), dict(dx=CONV["x"]),
               dict(dx=CONV["dy"]), dict(s=FAKE, dsi=FAKE), dict(ds=FAKE, dsi=FAKE), dict(ws=None), dict(ws=FAKE + 64)):
        assert call(f, CONV_BWD, CONV, kw) == sla.SLA_E_ARG, kw
    need = L.sla_short_conv_backward_workspace_bytes(100, 3, 1, 64, 4)
    assert need > 0 and call(f, CONV_BWD, CONV, dict(nbytes=need - 1)) == sla.SLA_E_WORKSPACE
    assert L.sla_short_conv_backward_workspace_bytes(100, 3, 1, 64, 9) == 0
    f = L.sla_step_short_conv
    for kw in (dict(slots=None), dict(slots=FAKE + 1), dict(pool=None), dict(pool=FAKE + 1), dict(y=None), dict(y=CONV["x"])):
        assert call(f, CONV_STEP, CONV, kw) == sla.SLA_E_ARG, kw
    assert call(f, CONV_STEP, CONV, dict(n=65537)) == sla.SLA_E_UNSUPPORTED
    assert call(f, CONV_STEP, CONV, dict(n=0, x=None, y=None)) == sla.SLA_OK


SCAN = dict(offsets=at(), n=100, W=3, order=None, dtype=1, D=64, G=2, N=16, sp=1, x=at(), ldx=64, d=at(), ldd=64, A=at(),
            B=at(), ldb=32, C=at(), ldc=40, skip=at(), z=at(), ldz=128, bias=at(), s=None, y=at(), so=None, dy=at(), ldy=64,
            ds=None, dx=at(), dd=at(), dA=at(), dB=at(), dC=at(), dskip=at(), dz=at(), dbias=at(), dsi=None, ws=at(), nbytes=BIG,
            stream=None, slots=at(), pool=at())
SCAN_ROWS = ["x", "ldx", "d", "ldd", "A", "B", "ldb", "C", "ldc", "skip", "z", "ldz", "bias"]
SCAN_HEAD = ["offsets", "n", "W", "order", "dtype", "D", "G", "N", "sp"]
SCAN_FWD = SCAN_HEAD + SCAN_ROWS + ["s", "y", "so", "ws", "nbytes", "stream"]
SCAN_BWD = SCAN_HEAD + SCAN_ROWS + ["s", "dy", "ldy", "ds", "dx", "dd", "dA", "dB", "dC", "dskip", "dz", "dbias", "dsi", "ws",
                                    "nbytes", "stream"]
SCAN_STEP = ["slots", "n", "W", "dtype", "D", "G", "N", "sp", "pool"] + SCAN_ROWS + ["y", "stream"]


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), "ARG"), (dict(n=2 ** 31 - 1), "ARG"), (dict(W=0), "ARG"), (dict(dtype=3), "ARG"), (dict(D=0), "ARG"),
    (dict(D=65537, G=1, ldx=1 << 20, ldd=1 << 20, ldz=1 << 20), "UNSUPPORTED"), (dict(G=0), "ARG"), (dict(G=3), "ARG"),
    (dict(N=0), "UNSUPPORTED"), (dict(N=65), "UNSUPPORTED"), (dict(W=2 ** 23), "UNSUPPORTED"),
    (dict(n=2 ** 31 - 2), "UNSUPPORTED"),
    (dict(D=65536, G=65536, ldx=65536, ldd=65536, ldz=65536, N=1, ldb=65536, ldc=65536), "UNSUPPORTED"),
    (dict(x=None), "ARG"), (dict(x=FAKE + 1), "ARG"), (dict(ldx=63), "ARG"), (dict(d=None), "ARG"), (dict(ldd=63), "ARG"),
    (dict(A=None), "ARG"), (dict(A=FAKE + 2), "ARG"), (dict(B=None), "ARG"), (dict(ldb=31), "ARG"), (dict(C=None), "ARG"),
    (dict(ldc=31), "ARG"), (dict(skip=FAKE + 2), "ARG"), (dict(z=FAKE + 1), "ARG"), (dict(ldz=63), "ARG"),
    (dict(bias=FAKE + 1), "ARG")])
def test_scan_refusals(L, kw, want):
    for f, order in ((L.sla_forward_selective_scan, SCAN_FWD), (L.sla_backward_selective_scan, SCAN_BWD),
                     (L.sla_step_selective_scan, SCAN_STEP)):
        assert call(f, order, SCAN, kw) == code(want)


def test_scan_refusals_of_one(L):
    f = L.sla_forward_selective_scan
    for kw in (dict(offsets=None), dict(offsets=FAKE + 2), dict(order=FAKE + 1), dict(y=None), dict(s=FAKE + 2),
               dict(so=FAKE + 2), dict(ws=None), dict(ws=FAKE + 16), *(dict(y=SCAN[k]) for k in ("x", "d", "B", "C", "z"))):
        assert call(f, SCAN_FWD, SCAN, kw) == sla.SLA_E_ARG, kw
    need = L.sla_selective_scan_workspace_bytes(100, 3, 1, 64, 2, 16)
    assert need > 0 and call(f, SCAN_FWD, SCAN, dict(nbytes=need - 1)) == sla.SLA_E_WORKSPACE
    rows = dict(x=None, d=None, B=None, C=None, z=None, y=None, ws=None, nbytes=0)
    assert call(f, SCAN_FWD, SCAN, dict(rows, n=0)) == sla.SLA_OK
    f = L.sla_backward_selective_scan
    for kw in (dict(dy=None), dict(ldy=63), *(dict([(k, None)]) for k in ("dx", "dd", "dA", "dB", "dC", "dz")),
               dict(dA=FAKE + 2), dict(dskip=FAKE + 2), dict(dbias=FAKE + 2), dict(dx=SCAN["x"]), dict(dd=SCAN["d"]),
               dict(dz=SCAN["z"]), dict(dB=SCAN["B"]), dict(dC=SCAN["C"]), dict(dx=SCAN["dy"]), dict(s=FAKE, dsi=FAKE),
               dict(ds=FAKE + 2), dict(ws=None), dict(ws=FAKE + 16)):
        assert call(f, SCAN_BWD, SCAN, kw) == sla.SLA_E_ARG, kw
    need = L.sla_selective_scan_backward_workspace_bytes(100, 3, 1, 64, 2, 16)
    assert need > 0 and call(f, SCAN_BWD, SCAN, dict(nbytes=need - 1)) == sla.SLA_E_WORKSPACE
    f = L.sla_step_selective_scan
    for kw in (dict(slots=None), dict(slots=FAKE + 1), dict(pool=None), dict(pool=FAKE + 2), dict(y=None), dict(y=SCAN["x"])):
        assert call(f, SCAN_STEP, SCAN, kw) == sla.SLA_E_ARG, kw
    assert call(f, SCAN_STEP, SCAN, dict(n=65537)) == sla.SLA_E_UNSUPPORTED
    assert call(f, SCAN_STEP, SCAN, dict(n=0, x=None, d=None, B=None, C=None, y=None)) == sla.SLA_OK
    for f in (L.sla_selective_scan_workspace_bytes, L.sla_selective_scan_backward_workspace_bytes):
        assert f(100, 3, 1, 64, 3, 16) == 0 and f(100, 3, 1, 64, 2, 65) == 0
        sizes = [f(n, 5, 1, 512, 1, 16) for n in (0, 1, 64, 1000, 100000, 10000000)]
        assert sizes[0] > 0 and sizes == sorted(sizes) and all(x % 256 == 0 for x in sizes)


NORM = dict(n=100, dtype=2, rtype=2, C=64, eps=1e-5, scale=1.0, act=2, x=at(), r=at(), g=at(), pw=at(), w=at(), y=at(), ro=at(),
            rstd=at(), ps=at(), dy=at(), dro=at(), dx=at(), dr=at(), dg=at(), dw=at(), dpw=at(), ws=at(), nbytes=BIG,
            stream=None)
NORM_FWD = ["n", "dtype", "rtype", "C", "eps", "scale", "act", "x", "r", "g", "pw", "w", "y", "ro", "rstd", "ps", "stream"]
NORM_BWD = ["n", "dtype", "rtype", "C", "scale", "act", "x", "ro", "g", "pw", "w", "rstd", "ps", "dy", "dro", "dx", "dr", "dg",
            "dw", "dpw", "ws", "nbytes", "stream"]


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), "ARG"), (dict(n=2 ** 31 - 1), "ARG"), (dict(dtype=3), "ARG"), (dict(rtype=1), "ARG"), (dict(rtype=-1), "ARG"),
    (dict(C=0), "ARG"), (dict(C=8193), "UNSUPPORTED"), (dict(act=3), "ARG"), (dict(scale=float("nan")), "ARG"),
    (dict(scale=float("inf")), "ARG"), (dict(x=None), "ARG"), (dict(x=FAKE + 1), "ARG"), (dict(ro=None), "ARG"),
    (dict(g=FAKE + 1), "ARG"), (dict(w=FAKE + 2), "ARG"), (dict(pw=FAKE + 2), "ARG"), (dict(rstd=None), "ARG"),
    (dict(ps=None), "ARG"), (dict(rtype=0, ro=FAKE + 2), "ARG")])
def test_norm_refusals(L, kw, want):
    assert call(L.sla_forward_residual_norm, NORM_FWD, NORM, kw) == code(want)
    assert call(L.sla_backward_residual_norm, NORM_BWD, NORM, kw) == code(want)


def test_norm_refusals_of_one(L):
    f = L.sla_forward_residual_norm
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(y=None), dict(r=FAKE + 1), *(dict(y=NORM[k]) for k in ("x", "g", "r")),
               dict(ro=NORM["x"]), dict(ro=NORM["g"]), dict(ro=NORM["y"])):
        assert call(f, NORM_FWD, NORM, kw) == sla.SLA_E_ARG, kw
    assert call(f, NORM_FWD, NORM, dict(n=0, x=None, y=None, ro=None, rstd=None)) == sla.SLA_OK
    f = L.sla_backward_residual_norm
    for kw in (dict(dy=None), dict(dx=None), dict(dg=None), dict(dro=FAKE + 1), dict(dw=FAKE + 2), dict(dx=NORM["x"]),
               dict(dx=NORM["dy"]), dict(dg=NORM["g"]), dict(dr=NORM["ro"]), dict(dx=NORM["dro"]), dict(ws=None),
               dict(ws=FAKE + 16)):
        assert call(f, NORM_BWD, NORM, kw) == sla.SLA_E_ARG, kw
    need = L.sla_residual_norm_backward_workspace_bytes(100, 2, 64)
    assert need > 0 and call(f, NORM_BWD, NORM, dict(nbytes=need - 1)) == sla.SLA_E_WORKSPACE
    assert L.sla_residual_norm_backward_workspace_bytes(100, 2, 8193) == 0


def test_one_output_for_two_gradients_is_refused(L):
    for kw in (dict(dd=SCAN["dx"]), dict(dz=SCAN["dd"]), dict(dC=SCAN["dB"]), dict(dB=SCAN["dz"])):
        assert call(L.sla_backward_selective_scan, SCAN_BWD, SCAN, kw) == sla.SLA_E_ARG, kw
    for kw in (dict(dr=NORM["dx"]), dict(dg=NORM["dx"]), dict(dg=NORM["dr"])):
        assert call(L.sla_backward_residual_norm, NORM_BWD, NORM, kw) == sla.SLA_E_ARG, kw


# ------------------------------------------------------------------ the binding
def test_conv_binding():
    import torch

    x, w, off = torch.zeros(6, 8), torch.zeros(8, 4), torch.tensor([0, 6], dtype=torch.int32)
    ok = dict(x=x, weight=w, offsets=off)
    for kw in (dict(x=x[0]), dict(x=torch.zeros(8, 6).t()), dict(x=torch.zeros(1, 8).expand(6, 8)), dict(weight=w[:7]),
               dict(weight=w.half()), dict(weight=w[0]), dict(bias=w), dict(activation="gelu"), dict(offsets=off.long()),
               dict(order=off), dict(state=torch.zeros(1, 4, 8)), dict(state=torch.zeros(1, 3, 8).half()), dict(y=x.half()),
               dict(final_state=torch.zeros(2, 3, 8))):
        with pytest.raises(ValueError):
            sla.forward_short_conv(**{**ok, **kw})
    for kw in (dict(dy=x[:5]), dict(dy=x.half()), dict(dy=x, dstate=x), dict(dy=x, dx=x.half())):
        with pytest.raises(ValueError):
            sla.backward_short_conv(**ok, **kw)
    pool, slots = torch.zeros(4, 3, 8), torch.zeros(6, dtype=torch.int32)
    for kw in (dict(state=pool[0], slots=slots), dict(state=pool[:0], slots=slots), dict(state=pool.half(), slots=slots),
               dict(state=pool, slots=slots.long()), dict(state=pool, slots=slots[:5]), dict(state=pool, slots=slots, y=pool)):
        with pytest.raises(ValueError):
            sla.step_short_conv(x=x, weight=w, **kw)
    with pytest.raises((ValueError, sla.SlaError)):   # host memory
        sla.forward_short_conv(**ok)


def test_scan_binding():
    import torch

    n, D, N, G = 6, 8, 4, 2
    x, A, B = torch.zeros(n, D), torch.zeros(D, N), torch.zeros(n, G, N)
    off = torch.tensor([0, n], dtype=torch.int32)
    ok = dict(x=x, delta=x, A=A, B=B, C=B, offsets=off)
    bad = (dict(x=x[0]), dict(x=x.t()), dict(delta=x[:5]), dict(delta=x.half()), dict(A=A[:7]), dict(A=A.half()), dict(B=B[:, 0]),
           dict(B=B.transpose(1, 2)), dict(C=B[:, :1]), dict(C=B.half()), dict(B=torch.zeros(n, 3, N), C=torch.zeros(n, 3, N)),
           dict(skip=A), dict(delta_bias=x[0].half()), dict(z=x[:, :4]), dict(z=x.half()))
    more = (dict(offsets=off[:1]), dict(order=off), dict(state=torch.zeros(2, D, N)), dict(y=x.half()),
            dict(final_state=torch.zeros(1, N, D)))
    for kw in (*bad, *more):
        with pytest.raises(ValueError):
            sla.forward_selective_scan(**{**ok, **kw})
    for kw in (dict(dy=x[:5]), dict(dy=x, dstate=x), dict(dy=x, out=[x]), dict(dy=x, out=[x, x, B, B, x]),
               dict(dy=x, out=[x, x, B, x, None])):
        with pytest.raises(ValueError):
            sla.backward_selective_scan(**ok, **kw)
    pool, slots = torch.zeros(4, D, N), torch.zeros(n, dtype=torch.int32)
    rows = {k: v for k, v in ok.items() if k != "offsets"}
    for kw in bad:
        with pytest.raises(ValueError):
            sla.step_selective_scan(pool, slots, **{**rows, **kw})
    for kw in (dict(state=pool[0]), dict(state=pool.half()), dict(slots=slots[:5]), dict(slots=slots.long()), dict(y=A)):
        with pytest.raises(ValueError):
            sla.step_selective_scan(**{**dict(state=pool, slots=slots), **rows, **kw})
    with pytest.raises(sla.SlaError):
        sla.forward_selective_scan(x, x, torch.zeros(D, 65), torch.zeros(n, 1, 65), torch.zeros(n, 1, 65), off)


def test_norm_binding():
    import torch

    x, w, s = torch.zeros(6, 8), torch.zeros(8), torch.zeros(6)
    for kw in (dict(x=x[0]), dict(x=x.t()), dict(residual=x[:5]), dict(residual=x.half()), dict(weight=w.half()),
               dict(post_weight=w[:7]), dict(gate=x.half()), dict(activation="tanh"), dict(y=x.half()),
               dict(residual_out=x.half())):
        with pytest.raises(ValueError):
            sla.forward_residual_norm(**{**dict(x=x, residual=x), **kw})
    ok = dict(x=x, residual_out=x, dy=x, rstd=s)
    for kw in (dict(dy=x.half()), dict(rstd=s[:5]), dict(post_weight=w), dict(post_rstd=s), dict(dresidual_out=x.half()),
               dict(dx=x.half()), dict(dresidual=x.half())):
        with pytest.raises(ValueError):
            sla.backward_residual_norm(**{**ok, **kw})


# ------------------------------------------------------------------ the references
def test_conv_reference_is_torch():
    import torch

    gen = torch.Generator().manual_seed(0)
    n, C, K = 11, 6, 4
    x, w = (torch.randn(*s, generator=gen, dtype=torch.float64, requires_grad=True) for s in ((n, C), (C, K)))
    b, st = (torch.randn(*s, generator=gen, dtype=torch.float64, requires_grad=True) for s in ((C,), (1, K - 1, C)))
    dy, ds = torch.randn(n, C, generator=gen, dtype=torch.float64), torch.randn(1, K - 1, C, generator=gen, dtype=torch.float64)
    full = torch.cat([st[0], x])
    y = torch.nn.functional.silu(torch.nn.functional.conv1d(full.t()[None], w[:, None], b, groups=C)[0].t())
    ((y * dy).sum() + (full[-(K - 1):] * ds[0]).sum()).backward()
    num = lambda t: t.detach().numpy()  # noqa: E731
    ry, rs = space_ref.conv_forward_ref(num(x), num(w), [0, n], num(b), "silu", state=num(st))
    assert np.abs(ry - num(y)).max() < 1e-13 and np.array_equal(rs[0], num(x)[-(K - 1):])
    got = space_ref.conv_backward_ref(num(x), num(w), [0, n], num(dy), num(b), "silu", state=num(st), dstate=num(ds))
    for a, e in zip(got, (x.grad, w.grad, b.grad, st.grad)):
        assert np.abs(a - num(e)).max() < 1e-12


def test_scan_reference_is_torch():
    import torch

    gen = torch.Generator().manual_seed(1)
    n, D, N, G = 9, 6, 3, 2
    new = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    t = dict(x=new(n, D), delta=new(n, D), A=-new(D, N).abs(), B=new(n, G, N), C=new(n, G, N), skip=new(D), z=new(n, D),
             bias=new(D), state=new(1, D, N))
    dy, ds = new(n, D), new(1, D, N)
    v = {k: x.clone().requires_grad_(True) for k, x in t.items()}
    dt = torch.nn.functional.softplus(v["delta"] + v["bias"])
    h, ys = v["state"][0], []
    for i in range(n):
        Bi, Ci = (v[k][i].repeat_interleave(D // G, 0) for k in ("B", "C"))
        h = torch.exp(dt[i][:, None] * v["A"]) * h + (dt[i] * v["x"][i])[:, None] * Bi
        ys.append((Ci * h).sum(-1) + v["skip"] * v["x"][i])
    y = torch.stack(ys) * torch.nn.functional.silu(v["z"])
    ((y * dy).sum() + (h * ds[0]).sum()).backward()
    num = lambda x: x.detach().numpy()  # noqa: E731
    args = [num(t[k]) for k in ("x", "delta", "A", "B", "C")]
    kw = dict(skip=num(t["skip"]), z=num(t["z"]), delta_bias=num(t["bias"]), delta_softplus=True, state=num(t["state"]))
    ry, rs = space_ref.scan_forward_ref(*args, [0, n], **kw)
    assert np.abs(ry - num(y)).max() < 1e-12 and np.abs(rs[0] - num(h)).max() < 1e-12
    got = space_ref.scan_backward_ref(*args, [0, n], num(dy), dstate=num(ds), **kw)
    for a, k in zip(got, ("x", "delta", "A", "B", "C", "skip", "z", "bias", "state")):
        assert np.abs(a - num(v[k].grad)).max() < 1e-11, k


def test_scan_reference_of_constant_steps_is_a_power():
    """One channel, one state, constant input: h_t = u (1 - a^t) / (1 - a)."""
    n = 7
    one = np.ones((n, 1))
    y, h = space_ref.scan_forward_ref(2 * one, 0.5 * one, np.array([[-1.0]]), one[:, :, None], 3 * one[:, :, None], [0, n])
    a = np.exp(-0.5)
    want = (1 - a ** np.arange(1, n + 1)) / (1 - a)
    assert np.abs(y[:, 0] - 3 * want).max() < 1e-13 and abs(h[0, 0, 0] - want[-1]) < 1e-13


def test_norm_reference_is_torch():
    import torch

    gen = torch.Generator().manual_seed(2)
    new = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64, requires_grad=True)  # noqa: E731
    n, C = 5, 7
    x, r, g, w, pw = new(n, C), new(n, C), new(n, C), new(C), new(C)
    dy, do = new(n, C).detach(), new(n, C).detach()
    rms = lambda v: v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
    ro = r + 0.3 * torch.nn.functional.silu(g) * rms(x) * pw
    y = rms(ro) * w
    ((y * dy).sum() + (ro * do).sum()).backward()
    num = lambda t: t.detach().numpy()  # noqa: E731
    kw = dict(weight=num(w), post_weight=num(pw), gate=num(g), activation="silu", scale=0.3)
    ry, rr, rstd, ps = space_ref.rnorm_forward_ref(num(x), num(r), **kw)
    assert np.abs(ry - num(y)).max() < 1e-13 and np.abs(rr - num(ro)).max() < 1e-13
    got = space_ref.rnorm_backward_ref(num(x), rr, num(dy), rstd, post_rstd=ps, dresidual_out=num(do), **kw)
    for a, e in zip(got, (x.grad, r.grad, w.grad, pw.grad, g.grad)):
        assert np.abs(a - num(e)).max() < 1e-12


def test_step_references_are_the_forwards():
    rng = np.random.default_rng(3)
    perm = np.array([0, 4, 1, 5, 2, 6, 3, 7, 8])
    slots = np.where(perm < 4, 2, 0)
    x, w = rng.standard_normal((9, 5)), rng.standard_normal((5, 3))
    y, S = space_ref.conv_forward_ref(x, w, [0, 4, 9])
    sy, pool = space_ref.conv_step_ref(np.zeros((3, 2, 5)), slots, x[perm], w)
    assert np.array_equal(sy, y[perm]) and np.array_equal(pool[2], S[0]) and np.array_equal(pool[0], S[1])
    d, A, B, C = rng.random((9, 5)), -rng.random((5, 2)), rng.standard_normal((9, 1, 2)), rng.standard_normal((9, 1, 2))
    y, S = space_ref.scan_forward_ref(x, d, A, B, C, [0, 4, 9])
    sy, pool = space_ref.scan_step_ref(np.zeros((3, 5, 2)), slots, x[perm], d[perm], A, B[perm], C[perm])
    assert np.allclose(sy, y[perm], atol=1e-14) and np.allclose(pool[2], S[0]) and np.allclose(pool[0], S[1])
