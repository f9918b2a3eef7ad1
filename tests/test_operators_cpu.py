"""CPU tests of the gated delta rule and of group normalisation: what the entry points and the
binding refuse (all of it before anything is launched), and their float64 references against other
forms of the same operators and against differences."""
from __future__ import annotations

import os

import numpy as np
import pytest

from oracle import delta_ref
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


DELTA = dict(offsets=FAKE, n=100, W=3, order=None, dtype=1, hk=2, h=4, dk=64, dv=32, scale=0.125, q=FAKE, k=FAKE, v=FAKE,
             g=FAKE, beta=FAKE, state=None, dout=FAKE, dstate=None, o=FAKE, state_out=None, dq=FAKE, dk_out=FAKE,
             dv_out=FAKE, dg=FAKE, dbeta=FAKE, dstate_in=None, ws=FAKE, nbytes=BIG, stream=None, slots=FAKE, pool=FAKE)
SIZES = ["offsets", "n", "W", "order", "dtype", "hk", "h", "dk", "dv", "scale", "q", "k", "v", "g", "beta", "state"]
FORWARD = SIZES + ["o", "state_out", "ws", "nbytes", "stream"]
BACKWARD = SIZES + ["dout", "dstate", "dq", "dk_out", "dv_out", "dg", "dbeta", "dstate_in", "ws", "nbytes", "stream"]
STEP = ["slots", "n", "W", "dtype", "hk", "h", "dk", "dv", "scale", "pool", "q", "k", "v", "g", "beta", "o", "stream"]

BAD_SIZES = [(dict(n=-1), "ARG"), (dict(n=2 ** 31 - 1), "ARG"), (dict(W=0), "ARG"), (dict(dtype=3), "ARG"),
             (dict(dtype=-1), "ARG"), (dict(hk=0), "ARG"), (dict(hk=3), "ARG"), (dict(h=0), "ARG"),
             (dict(hk=1, h=65536), "UNSUPPORTED"), (dict(dk=8), "UNSUPPORTED"), (dict(dk=40), "UNSUPPORTED"),
             (dict(dk=144), "UNSUPPORTED"), (dict(dv=0), "UNSUPPORTED"), (dict(dv=24), "UNSUPPORTED"),
             (dict(dv=272), "UNSUPPORTED"), (dict(n=2 ** 31 - 2), "UNSUPPORTED"), (dict(W=2 ** 23), "UNSUPPORTED"),
             (dict(scale=float("nan")), "ARG"), (dict(scale=float("inf")), "ARG")]


def code(name):
    return getattr(sla, "SLA_E_" + name)


@pytest.mark.parametrize("kw,want", BAD_SIZES)
def test_delta_sizes(L, kw, want):
    for f, order in ((L.sla_forward_delta, FORWARD), (L.sla_backward_delta, BACKWARD), (L.sla_step_delta, STEP)):
        assert call(f, order, DELTA, kw) == code(want)
    if "scale" not in kw:
        a = {**DELTA, **kw}
        sizes = [a[x] for x in ("n", "W", "dtype", "hk", "h", "dk", "dv")]
        assert L.sla_delta_workspace_bytes(*sizes) == 0 and L.sla_delta_backward_workspace_bytes(*sizes) == 0


def test_delta_pointers(L):
    for f, order, rows, other in (
            (L.sla_forward_delta, FORWARD, ["q", "k", "v", "o"], ["g", "beta"]),
            (L.sla_backward_delta, BACKWARD, ["q", "k", "v", "dout", "dq", "dk_out", "dv_out"], ["g", "beta", "dg", "dbeta"]),
            (L.sla_step_delta, STEP, ["q", "k", "v", "o", "pool"], ["g", "beta", "slots"])):
        for name in rows:
            assert call(f, order, DELTA, {name: None}) == sla.SLA_E_ARG, name
            assert call(f, order, DELTA, {name: FAKE + 8}) == sla.SLA_E_ARG, name
        for name in other:
            assert call(f, order, DELTA, {name: None}) == sla.SLA_E_ARG, name
            assert call(f, order, DELTA, {name: FAKE + 2}) == sla.SLA_E_ARG, name
    for f, order, states in ((L.sla_forward_delta, FORWARD, ["state", "state_out"]),
                             (L.sla_backward_delta, BACKWARD, ["state", "dstate", "dstate_in"])):
        for name in ["order", *states]:
            assert call(f, order, DELTA, {name: FAKE + 1}) == sla.SLA_E_ARG, name
        assert call(f, order, DELTA, dict(offsets=None)) == sla.SLA_E_ARG
        assert call(f, order, DELTA, dict(ws=None)) == sla.SLA_E_ARG
        assert call(f, order, DELTA, dict(ws=FAKE + 16)) == sla.SLA_E_ARG
        need = (L.sla_delta_workspace_bytes if order is FORWARD else L.sla_delta_backward_workspace_bytes)(
            100, 3, 1, 2, 4, 64, 32)
        assert need > 0 and call(f, order, DELTA, dict(nbytes=need - 1)) == sla.SLA_E_WORKSPACE
        # no rows and no state to hand on: nothing to do, nothing launched
        assert call(f, order, DELTA, dict(n=0, q=None, k=None, v=None, o=None, ws=None, nbytes=0)) == sla.SLA_OK
    assert call(L.sla_step_delta, STEP, DELTA, dict(n=0, q=None, o=None)) == sla.SLA_OK


def test_step_rows(L):
    assert call(L.sla_step_delta, STEP, DELTA, dict(n=65537)) == sla.SLA_E_UNSUPPORTED


NORM = dict(offsets=FAKE, n=100, W=3, dtype=2, C=64, G=4, eps=1e-5, act=2, x=FAKE, w=FAKE, b=FAKE, y=FAKE, dy=FAKE,
            mean=FAKE, rstd=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, nbytes=BIG, stream=None)
NORM_FORWARD = ["offsets", "n", "W", "dtype", "C", "G", "eps", "act", "x", "w", "b", "y", "mean", "rstd", "ws", "nbytes",
                "stream"]
NORM_BACKWARD = ["offsets", "n", "W", "dtype", "C", "G", "act", "x", "w", "b", "dy", "mean", "rstd", "dx", "dw", "db", "ws",
                 "nbytes", "stream"]


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), "ARG"), (dict(W=0), "ARG"), (dict(W=-1), "ARG"), (dict(offsets=None), "ARG"), (dict(dtype=3), "ARG"),
    (dict(C=0), "ARG"), (dict(G=0), "ARG"), (dict(G=3), "ARG"), (dict(act=3), "ARG"), (dict(act=-1), "ARG"),
    (dict(C=4100, G=1), "UNSUPPORTED"), (dict(G=32), "UNSUPPORTED"), (dict(C=6, G=1), "UNSUPPORTED"),
    (dict(n=2 ** 31 - 2), "UNSUPPORTED"), (dict(W=2 ** 22), "UNSUPPORTED"), (dict(offsets=FAKE + 2), "ARG"),
    (dict(w=FAKE + 4), "ARG"), (dict(b=FAKE + 8), "ARG"), (dict(x=FAKE + 8), "ARG"), (dict(x=None), "ARG"),
    (dict(mean=None), "ARG"), (dict(rstd=FAKE + 2), "ARG"), (dict(ws=None), "ARG"), (dict(ws=FAKE + 64), "ARG"),
    (dict(nbytes=0), "WORKSPACE")])
def test_norm_refusals(L, kw, want):
    assert call(L.sla_forward_group_norm, NORM_FORWARD, NORM, kw) == code(want)
    assert call(L.sla_backward_group_norm, NORM_BACKWARD, NORM, kw) == code(want)


def test_norm_refusals_of_one(L):
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(L.sla_forward_group_norm, NORM_FORWARD, NORM, dict(eps=eps)) == sla.SLA_E_ARG
    for kw in (dict(y=None), dict(y=FAKE + 8)):
        assert call(L.sla_forward_group_norm, NORM_FORWARD, NORM, kw) == sla.SLA_E_ARG
    for kw in (dict(dy=None), dict(dx=None), dict(dx=FAKE + 4), dict(dw=FAKE + 1), dict(db=FAKE + 2)):
        assert call(L.sla_backward_group_norm, NORM_BACKWARD, NORM, kw) == sla.SLA_E_ARG
    empty = dict(n=0, W=0, offsets=None, x=None, y=None, mean=None, rstd=None)
    assert call(L.sla_forward_group_norm, NORM_FORWARD, NORM, empty) == sla.SLA_OK
    assert L.sla_group_norm_workspace_bytes(100, 3, 2, 64, 3) == 0
    assert L.sla_group_norm_backward_workspace_bytes(100, 0, 2, 64, 4) > 0


def test_workspaces_grow_with_the_rows(L):
    for f in (L.sla_delta_workspace_bytes, L.sla_delta_backward_workspace_bytes):
        for dtype in range(3):
            sizes = [f(n, 5, dtype, 2, 4, 64, 64) for n in (0, 1, 64, 1000, 100000, 10000000)]
            assert sizes[0] > 0 and sizes == sorted(sizes) and sizes[-1] > 1 << 32
            assert all(x % 256 == 0 for x in sizes)


# ------------------------------------------------------------------ the binding
def delta_rows(n=6, hk=1, h=2, dk=32, dv=16):
    import torch

    return dict(q=torch.zeros(n, hk, dk), k=torch.zeros(n, hk, dk), v=torch.zeros(n, h, dv), g=torch.zeros(n, h),
                beta=torch.zeros(n, h), offsets=torch.tensor([0, n], dtype=torch.int32))


@pytest.mark.parametrize("change", [
    dict(q=lambda t: t["q"][:, 0]), dict(q=lambda t: t["q"].transpose(0, 2)), dict(k=lambda t: t["k"][:5]),
    dict(k=lambda t: t["k"].half()), dict(v=lambda t: t["v"][:5]), dict(v=lambda t: t["v"].double()),
    dict(g=lambda t: t["g"].half()), dict(g=lambda t: t["g"][:, :1]), dict(beta=lambda t: t["beta"].t()),
    dict(offsets=lambda t: t["offsets"].long()), dict(offsets=lambda t: t["offsets"][:1]),
    dict(order=lambda t: t["offsets"]), dict(state=lambda t: t["q"]), dict(out=lambda t: t["q"]),
    dict(final_state=lambda t: t["q"])])
def test_forward_binding(change):
    t = delta_rows()
    kw = {**t, **{name: f(t) for name, f in change.items()}}
    with pytest.raises(ValueError):
        sla.forward_delta(**kw)


def test_other_bindings():
    import torch

    t = delta_rows()
    dout = torch.zeros_like(t["v"])
    three = dict(t, q=torch.zeros(6, 3, 32), k=torch.zeros(6, 3, 32))
    for kw in (dict(t, dout=dout.half()), dict(t, dout=dout, dstate=dout), dict(t, dout=dout, out=[dout]),
               dict(t, dout=dout, out=[dout] * 5), dict(three, dout=dout)):
        with pytest.raises(ValueError):
            sla.backward_delta(**kw)
    rows = {x: t[x] for x in ("q", "k", "v", "g", "beta")}
    pool, slots = torch.zeros(4, 2, 32, 16), torch.zeros(6, dtype=torch.int32)
    for kw in (dict(state=pool[0], slots=slots), dict(state=pool[:0], slots=slots), dict(state=pool.half(), slots=slots),
               dict(state=pool, slots=slots.long()), dict(state=pool, slots=slots[:5]),
               dict(state=pool, slots=slots, out=pool)):
        with pytest.raises(ValueError):
            sla.step_delta(**kw, **rows)
    x, off = torch.zeros(6, 32), t["offsets"]
    stat = torch.zeros(6, 4)
    for kw in (dict(x=x[0], groups=4), dict(x=x.t(), groups=2), dict(x=x, groups=0), dict(x=x, groups=5),
               dict(x=x, groups=4, weight=x[0].half()), dict(x=x, groups=4, bias=x[0, :8]),
               dict(x=x, groups=4, activation="gelu"), dict(x=x, groups=4, offsets=off.long()),
               dict(x=x, groups=4, y=x.half()), dict(x=x, groups=4, mean=x)):
        with pytest.raises(ValueError):
            sla.forward_group_norm(**kw)
    for kw in (dict(dy=x.half()), dict(dy=x, mean=stat[:1]), dict(dy=x, rstd=stat.double()), dict(dy=x, dx=x.half())):
        with pytest.raises(ValueError):
            sla.backward_group_norm(**{**dict(x=x, groups=4, mean=stat, rstd=stat), **kw})


def test_sizes_that_are_not_supported_raise():
    import torch

    t = delta_rows(dk=24)
    with pytest.raises(sla.SlaError):
        sla.forward_delta(**t)
    with pytest.raises(sla.SlaError):
        sla.backward_delta(**t, dout=torch.zeros_like(t["v"]))
    with pytest.raises(sla.SlaError):
        sla.forward_group_norm(torch.zeros(6, 32), 16)


def test_tensors_in_host_memory_are_refused():
    import torch

    t = delta_rows()
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        sla.forward_delta(**t)
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        sla.forward_group_norm(torch.zeros(6, 32), 4)


# ------------------------------------------------------------------ the references
def rows(n, hk, h, dk, dv, seed=0):
    rng = np.random.default_rng(seed)
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    return dict(q=unit(rng.standard_normal((n, hk, dk))), k=unit(rng.standard_normal((n, hk, dk))),
                v=rng.standard_normal((n, h, dv)), g=-rng.random((n, h)), beta=rng.random((n, h)))


def test_forward_reference_is_its_closed_form():
    """One window, one head, from a state: o = scale (q' S0 + P u), u = beta (T (v - k' S0))."""
    r = rows(20, 1, 1, 8, 6)
    q, k, v = (r[x][:, 0] for x in "qkv")
    g, beta = r["g"][:, 0], r["beta"][:, 0]
    S0 = np.random.default_rng(1).standard_normal((1, 1, 8, 6))
    gam = np.cumsum(g)
    D = np.tril(np.exp(gam[:, None] - gam[None]))
    A = np.tril(D * (k @ k.T), -1) * beta[None]
    resid = np.linalg.solve(np.eye(20) + A, v - np.exp(gam)[:, None] * (k @ S0[0, 0]))
    u = beta[:, None] * resid
    o = 0.3 * (np.exp(gam)[:, None] * (q @ S0[0, 0]) + (D * (q @ k.T)) @ u)
    S = np.exp(gam[-1]) * S0[0, 0] + (np.exp(gam[-1] - gam)[:, None] * k).T @ u
    got, state = delta_ref.delta_forward_ref(**r, offsets=[0, 20], scale=0.3, state=S0)
    # sums of 20 terms in 53 bits
    assert np.abs(got[:, 0] - o).max() < 1e-13 and np.abs(state[0, 0] - S).max() < 1e-13


def test_forward_reference_without_keys_in_common_is_linear_attention():
    """Orthogonal keys, no decay, beta 1: nothing is taken back, S = sum k v."""
    n = 6
    q, v = np.random.default_rng(2).standard_normal((2, n, 1, n))
    o, S = delta_ref.delta_forward_ref(q, np.eye(n)[:, None], v, np.zeros((n, 1)), np.ones((n, 1)), [0, n], 1.0)
    assert np.abs(S[0, 0] - v[:, 0]).max() < 1e-14
    assert np.abs(o[:, 0] - np.tril(q[:, 0]) @ v[:, 0]).max() < 1e-13


def test_step_reference_is_the_forward():
    r = rows(9, 1, 2, 8, 4)
    o, S = delta_ref.delta_forward_ref(**r, offsets=[0, 4, 9], scale=0.5)
    perm = np.array([0, 4, 1, 5, 2, 6, 3, 7, 8])
    slots = np.where(perm < 4, 2, 0)
    so, pool = delta_ref.delta_step_ref(np.zeros((3, 2, 8, 4)), slots, **{x: t[perm] for x, t in r.items()}, scale=0.5)
    assert np.array_equal(so, o[perm]) and np.array_equal(pool[2], S[0]) and np.array_equal(pool[0], S[1])


def test_backward_reference_by_differences():
    r = rows(7, 1, 2, 4, 3, seed=3)
    rng = np.random.default_rng(4)
    x = dict(r, state=rng.standard_normal((2, 2, 4, 3)))
    order, off = rng.permutation(7), [0, 5, 7]
    dout, dst = rng.standard_normal((7, 2, 3)), rng.standard_normal((2, 2, 4, 3))

    def loss(x):
        o, S = delta_ref.delta_forward_ref(**x, offsets=off, scale=0.7, order=order)
        return (o * dout).sum() + (S * dst).sum()

    grads = delta_ref.delta_backward_ref(*(x[t] for t in ("q", "k", "v", "g", "beta")), off, dout, 0.7, x["state"], dst,
                                         order)
    for name, grad in zip(("q", "k", "v", "g", "beta", "state"), grads):
        d, h = rng.standard_normal(x[name].shape), 1e-5
        up, down = (loss({**x, name: x[name] + s * h * d}) for s in (1, -1))
        # h^2 and 2^-53 / h of losses near 10
        assert abs((up - down) / (2 * h) - (grad * d).sum()) < 1e-7, name


@pytest.mark.parametrize("activation", ["none", "relu", "silu"])
def test_norm_reference_is_torch(activation):
    import torch

    gen = torch.Generator().manual_seed(0)
    x = torch.randn(12, 24, generator=gen, dtype=torch.float64, requires_grad=True)
    w, b = (torch.randn(24, generator=gen, dtype=torch.float64, requires_grad=True) for _ in range(2))
    off = [0, 5, 5, 12]
    act = {"none": lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu}[activation]
    parts = [torch.nn.functional.group_norm(x[a:e].t()[None], 3, w, b, 1e-5)[0].t() for a, e in zip(off, off[1:]) if e > a]
    y = act(torch.cat(parts))
    dy = torch.randn(12, 24, generator=gen, dtype=torch.float64)
    y.backward(dy)
    num = lambda t: t.detach().numpy()  # noqa: E731
    ry, mean, rstd = delta_ref.group_norm_forward_ref(num(x), 3, num(w), num(b), off, 1e-5, activation)
    assert np.abs(ry - num(y)).max() < 1e-12 and mean[1].max() == 0
    got = delta_ref.group_norm_backward_ref(num(x), 3, num(dy), mean, rstd, num(w), num(b), off, activation)
    for a, e in zip(got, (x.grad, w.grad, b.grad)):
        assert np.abs(a - num(e)).max() < 1e-11


def test_the_declared_activations_are_the_binding_s():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sla.h")).read()
    for name, value in sla.ACTIVATIONS.items():
        assert f"SLA_ACT_{name.upper()} = {value}" in text
