"""The gated delta rule against its float64 reference.

Tolerances.  The kernels keep sums and states in fp32 and matrix-core operands in two fp16
terms, 2^-22 of an operand.  A row's result passes at most ten such operands (state, T, y, u,
P, forward and again backward), each off by 2^-22 of the largest value it is summed with: 10 *
2^-22 = 2.4e-6 of the largest result, times 4 for results that are differences of larger terms
(the residual v - S^T k, the decays' gradients): 1e-5, the bar of every fp32 result here.  A
16-bit result is off by that and by half a step of its own value.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import delta_ref
from tests.gpu_util import torch_dtype

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FP32_BAR = 1e-5
# bf16 outputs alone (nothing else comes from them): q S0 + P u with S0, P and u in one fp16 term each,
# off by half a step, 2^-11: 3 * 2^-11 of the largest result, three eighths of bf16's own half step.
OUT_BAR = {"f32": FP32_BAR, "f16": FP32_BAR, "bf16": 3 * 2.0 ** -11}


@pytest.fixture(scope="module")
def sla():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2401_00912_amd import sla as S

    S.lib()
    return S


def close(got, ref, dtype, name, bar=FP32_BAR):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, name
    real = ~np.isnan(ref)
    assert np.isfinite(got[real]).all(), f"{name} is not finite"
    top = np.abs(ref[real]).max() if real.any() else 0.0
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0
    limit = HALF_STEP[dtype] * np.abs(ref[real]) + bar * max(top, 1e-30) + tiny
    worst = np.max(np.abs(got[real] - ref[real]) / limit) if real.any() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times its limit"


class Case:
    """Rows as a layer makes them (normalised keys, log decays of slow and fast heads), rounded to dtype, on
    the device and in float64."""

    def __init__(self, lengths, hk, h, dk, dv, dtype, seed=0, state=False, behind=0, order=False, grads=False):
        import torch

        gen = torch.Generator().manual_seed(seed)
        n, w = int(sum(lengths)) + behind, len(lengths)
        self.n, self.w, self.dtype, self.scale = n, w, dtype, dk ** -0.5
        dt = torch_dtype(dtype)
        normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
        silu = torch.nn.functional.silu
        self.q, self.k = unit(silu(normal(n, hk, dk))).to(dt), unit(silu(normal(n, hk, dk))).to(dt)
        self.v = normal(n, h, dv).to(dt)
        rate = torch.exp(torch.rand(h, generator=gen) * 5 - 4)
        self.g = -rate * torch.nn.functional.softplus(normal(n, h))
        self.beta = torch.sigmoid(normal(n, h))
        self.state = 0.3 * normal(w, h, dk, dv) if state else None
        self.offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        self.order = torch.randperm(n, generator=gen).to(torch.int32) if order else None
        self.dout = normal(n, h, dv).to(dt) if grads else None
        self.dstate = normal(w, h, dk, dv) if grads and state else None

    def dev(self, name):
        import torch

        x = getattr(self, name)
        return None if x is None else (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).cuda()

    def wide(self, name):
        x = getattr(self, name)
        return None if x is None else x.numpy() if name == "order" else x.double().numpy()

    def forward_ref(self):
        return delta_ref.delta_forward_ref(*(self.wide(x) for x in ("q", "k", "v", "g", "beta")), self.offsets,
                                           self.scale, self.wide("state"), self.wide("order"))

    def forward(self, S, **kw):
        return S.forward_delta(*(self.dev(x) for x in ("q", "k", "v", "g", "beta", "offsets")), order=self.dev("order"),
                               state=self.dev("state"), **kw)


def check_forward(S, c):
    import torch

    out = torch.full_like(c.dev("v"), 7.0)
    o, st = c.forward(S, out=out)
    ro, rs = c.forward_ref()
    close(o, ro, c.dtype, "o", OUT_BAR[c.dtype])
    close(st, rs, "f32", "state")
    rest = np.isnan(ro).reshape(ro.shape)
    assert (o.double().cpu().numpy()[rest] == 7.0).all(), "rows in no window are left as they were"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 1, 32, 16), (2, 4, 64, 64), (1, 2, 128, 128), (3, 3, 16, 48),
                                        (1, 4, 96, 144), (2, 2, 48, 256), (1, 1, 112, 32)])
def test_forward_widths(sla, hk, h, dk, dv, dtype):
    check_forward(sla, Case([70, 1, 0, 64, 129, 17], hk, h, dk, dv, dtype, seed=dk + dv, state=dk % 32 == 0))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", [[1], [2], [15], [16], [17], [31], [32], [33], [48], [63], [64], [65], [127], [128],
                                     [129], [700], [0], [0, 0, 5, 0], [1] * 70, [64, 64, 64], [63, 65, 0, 1, 130]])
def test_forward_lengths(sla, lengths, dtype):
    check_forward(sla, Case(lengths, 1, 2, 32, 32, dtype, seed=len(lengths) + sum(lengths), state=len(lengths) % 2 == 0,
                            behind=3))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_order(sla, dtype):
    check_forward(sla, Case([40, 0, 90, 7, 64], 2, 4, 64, 32, dtype, seed=5, state=True, behind=6, order=True))


LONG = [[1100], [1024, 0, 1], [2500, 3, 1], [513, 1, 0, 2049, 512]]   # cut into parts of 512 rows


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", LONG)
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 2, 32, 32), (1, 1, 128, 80), (1, 1, 48, 16)])
def test_forward_long(sla, lengths, hk, h, dk, dv, dtype):
    check_forward(sla, Case(lengths, hk, h, dk, dv, dtype, seed=sum(lengths) + dk, state=len(lengths) > 1, behind=2,
                            order=dk == 48))


def test_forward_of_a_plan(sla):
    """Rows in any order with a window id each: a plan's offsets and perm."""
    import torch

    c = Case([50, 80, 3, 0, 66], 1, 2, 32, 32, "f16", seed=8)
    ids = np.repeat(np.arange(5), np.diff(c.offsets)).astype(np.int32)
    np.random.default_rng(1).shuffle(ids)
    plan = sla.build_segments(torch.from_numpy(ids).cuda(), num_windows=5)
    o, st = sla.forward_delta(*(c.dev(x) for x in ("q", "k", "v", "g", "beta")), plan.offsets, order=plan.perm)
    perm = np.argsort(ids, kind="stable")
    ro, rs = delta_ref.delta_forward_ref(*(c.wide(x) for x in ("q", "k", "v", "g", "beta")),
                                         np.concatenate([[0], np.cumsum(np.bincount(ids, minlength=5))]), c.scale,
                                         order=perm)
    close(o, ro, "f16", "o")
    close(st, rs, "f32", "state")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_forward_decays(sla, dtype):
    """No decay, fast decay, decays that forget everything (-infinity and what underflows) inside a chunk."""
    import torch

    c = Case([200, 64], 1, 2, 32, 32, dtype, seed=9, state=True)
    c.g[:, 0] = 0.0
    c.g[10:20, 0] = -30.0
    c.g[70, 0] = -torch.inf
    c.g[100, 1] = -torch.inf
    c.g[101, 1] = -torch.inf
    c.g[130, 1] = -200.0
    c.g[200, 1] = -torch.inf
    check_forward(sla, c)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_forward_scales(sla, dtype):
    """Keys, queries and values far from 1, a zero key, a zero beta, beta |k|^2 = 2."""
    import torch

    c = Case([150], 1, 2, 64, 32, dtype, seed=10)
    up = 256.0 if dtype == "f16" else 2.0 ** 20
    k = c.k.float()
    k[::3] *= up
    c.beta[::3] /= up * up
    k[1::3] /= 16.0
    c.k = k.to(c.k.dtype)
    c.k[7] = 0
    c.beta[9] = 0
    c.beta[11] = 2.0 / c.k[11].float().square().sum()
    c.q = (c.q.float() * 64.0).to(c.q.dtype)
    c.v = (c.v.float() * 100.0).to(c.v.dtype)
    check_forward(sla, c)


def test_forward_not_finite(sla):
    """A NaN or an infinity reaches only its own window, and v's only its own head and column."""
    import torch

    c = Case([70, 90, 80], 1, 2, 32, 32, "bf16", seed=11)
    clean, cs = c.forward(sla)
    c.v[75, 1, 3] = torch.nan
    c.k[170, 0, 5] = torch.inf
    bad, bs = c.forward(sla)
    want = torch.ones(clean.shape, dtype=torch.bool)
    want[75:160, 1, 3] = False
    want[170:240] = False
    # the rows of a 16 x 16 tile before row 75 share its products: column 3 may be lost from the chunk's start
    want[70:75, 1, 3] = False
    want[160:170] = False
    want = want.cuda()
    assert torch.equal(clean[want], bad[want])
    assert not torch.isfinite(bad[75:160, 1, 3].float()).any()
    assert torch.equal(cs[0], bs[0]) and torch.isfinite(bs[1][0]).all()
    cols = [x for x in range(32) if x != 3]
    assert torch.equal(cs[1][1][:, cols], bs[1][1][:, cols])


def test_forward_same_twice_and_in_place(sla):
    import torch

    c = Case([300, 5, 64], 2, 2, 64, 64, "bf16", seed=12, state=True)
    o, st = c.forward(sla)
    o2, st2 = c.forward(sla)
    assert torch.equal(o, o2) and torch.equal(st, st2)
    pool = c.dev("state")
    o3, st3 = sla.forward_delta(*(c.dev(x) for x in ("q", "k", "v", "g", "beta", "offsets")), state=pool, final_state=pool)
    assert torch.equal(o, o3) and torch.equal(st, pool) and st3 is pool


def test_forward_joins(sla):
    """A sequence in two calls, the state handed on, is the sequence in one call (to fp32 rounding: the
    chunks lie elsewhere)."""
    c = Case([230], 1, 2, 64, 32, "f32", seed=13)
    args = [c.dev(x) for x in ("q", "k", "v", "g", "beta")]
    import torch

    off = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    o, st = sla.forward_delta(*args, off(0, 230))
    a, s1 = sla.forward_delta(*(x[:101].contiguous() for x in args), off(0, 101))
    b, s2 = sla.forward_delta(*(x[101:].contiguous() for x in args), off(0, 129), state=s1)
    close(torch.cat([a, b]), o.double().cpu().numpy(), "f32", "o")
    close(s2, st.double().cpu().numpy(), "f32", "state")


# ------------------------------------------------------------------ gradients
GRADS = ("dq", "dk", "dv", "dg", "dbeta", "dstate_in")
# dq and dk of bf16 rows: three sums (the state, rows before, rows behind) of products with up to two
# operands in one fp16 term, each off by half a step, 2^-11: 6 * 2^-11 of the largest result if all were
# off that much to the same side; they are random, so a quarter of it.
OWN_BAR = {"f32": FP32_BAR, "f16": FP32_BAR, "bf16": 1.5 * 2.0 ** -11}


def check_backward(S, c):
    import torch

    outs = [torch.full_like(c.dev(x), 7.0) for x in ("q", "k", "v", "g", "beta")]
    got = S.backward_delta(*(c.dev(x) for x in ("q", "k", "v", "g", "beta", "offsets", "dout")), dstate=c.dev("dstate"),
                           order=c.dev("order"), state=c.dev("state"), out=outs)
    ref = delta_ref.delta_backward_ref(*(c.wide(x) for x in ("q", "k", "v", "g", "beta")), c.offsets, c.wide("dout"),
                                       c.scale, c.wide("state"), c.wide("dstate"), c.wide("order"))
    for name, x, r in zip(GRADS, got, ref):
        if x is None:
            assert name == "dstate_in" and c.state is None
            continue
        close(x, r, c.dtype if name in ("dq", "dk", "dv") else "f32", name,
              OWN_BAR[c.dtype] if name in ("dq", "dk") else FP32_BAR)
        assert (x.double().cpu().numpy()[np.isnan(r)] == 7.0).all(), f"{name}: rows in no window are left as they were"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 1, 32, 16), (2, 4, 64, 64), (1, 2, 128, 128), (3, 3, 16, 48),
                                        (1, 4, 96, 144), (2, 2, 48, 256), (1, 1, 112, 32)])
def test_backward_widths(sla, hk, h, dk, dv, dtype):
    check_backward(sla, Case([70, 1, 0, 64, 129, 17], hk, h, dk, dv, dtype, seed=dk + dv, state=dk % 32 == 0, grads=True))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", [[1], [2], [15], [16], [17], [32], [33], [63], [64], [65], [128], [129], [500], [0],
                                     [0, 0, 5, 0], [1] * 70, [64, 64, 64], [63, 65, 0, 1, 130]])
def test_backward_lengths(sla, lengths, dtype):
    check_backward(sla, Case(lengths, 1, 2, 32, 32, dtype, seed=len(lengths) + sum(lengths), state=len(lengths) % 2 == 0,
                             behind=3, grads=True))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", LONG)
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 2, 32, 32), (1, 1, 128, 80), (1, 1, 48, 16)])
def test_backward_long(sla, lengths, hk, h, dk, dv, dtype):
    check_backward(sla, Case(lengths, hk, h, dk, dv, dtype, seed=sum(lengths) + dk, state=len(lengths) > 1, behind=2,
                             order=dk == 48, grads=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_order(sla, dtype):
    check_backward(sla, Case([40, 0, 90, 7, 64], 2, 4, 64, 32, dtype, seed=5, state=True, behind=6, order=True,
                             grads=True))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_backward_decays(sla, dtype):
    import torch

    c = Case([200, 64], 1, 2, 32, 32, dtype, seed=9, state=True, grads=True)
    c.g[:, 0] = 0.0
    c.g[10:20, 0] = -30.0
    c.g[70, 0] = -torch.inf
    c.g[100, 1] = -torch.inf
    c.g[101, 1] = -torch.inf
    c.g[130, 1] = -200.0
    c.g[200, 1] = -torch.inf
    check_backward(sla, c)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_backward_scales(sla, dtype):
    """Queries and output gradients far from 1, a zero key, a zero beta, beta |k|^2 = 2."""
    c = Case([150], 1, 2, 64, 32, dtype, seed=10, grads=True)
    c.k[7] = 0
    c.beta[9] = 0
    c.beta[11] = 2.0 / c.k[11].float().square().sum()
    c.k = (c.k.float() * 8.0).to(c.k.dtype)
    c.beta /= 64.0
    c.q = (c.q.float() * 64.0).to(c.q.dtype)
    c.dout = (c.dout.float() / 16.0).to(c.dout.dtype)
    check_backward(sla, c)


def test_backward_by_differences(sla):
    """The gradients against differences of the forward kernel itself, in directions over every input."""
    import torch

    c = Case([70, 33], 1, 2, 32, 32, "f32", seed=21, state=True, grads=True)
    x = {n: c.dev(n).double() for n in ("q", "k", "v", "g", "beta", "state")}
    off, dout, dst = c.dev("offsets"), c.dev("dout"), c.dev("dstate")

    def loss(y):
        y = {n: t.float() for n, t in y.items()}
        o, st = sla.forward_delta(*(y[n] for n in ("q", "k", "v", "g", "beta")), off, state=y["state"])
        return float((o.double() * dout.double()).sum() + (st.double() * dst.double()).sum())

    grads = sla.backward_delta(*(x[n].float() for n in ("q", "k", "v", "g", "beta")), off, dout, dstate=dst,
                               state=x["state"].float())
    gen = torch.Generator().manual_seed(4)
    for name, grad in zip(("q", "k", "v", "g", "beta", "state"), grads):
        d = torch.randn(x[name].shape, generator=gen, dtype=torch.float64).cuda()
        h = 1e-3
        up, down = ({**x, name: x[name] + s * h * d} for s in (1, -1))
        got, want = float((grad.double() * d).sum()), (loss(up) - loss(down)) / (2 * h)
        # the loss is off by 1e-6 of its terms' norm and the difference by its third derivative h^2
        norm = float((dout.double().norm() ** 2 + dst.double().norm() ** 2) ** 0.5)
        assert abs(got - want) <= 1e-6 * norm / h * 2 + 1e-3 * abs(want), name


def test_backward_same_twice(sla):
    import torch

    c = Case([300, 5, 64], 2, 4, 64, 64, "bf16", seed=12, state=True, grads=True)
    args = [c.dev(x) for x in ("q", "k", "v", "g", "beta", "offsets", "dout")]
    a = sla.backward_delta(*args, dstate=c.dev("dstate"), state=c.dev("state"))
    b = sla.backward_delta(*args, dstate=c.dev("dstate"), state=c.dev("state"))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------ row by row
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 1, 32, 16), (2, 4, 64, 64), (1, 2, 128, 128), (3, 3, 16, 48), (1, 2, 80, 256)])
def test_step(sla, hk, h, dk, dv, dtype):
    import torch

    c = Case([1] * 9, hk, h, dk, dv, dtype, seed=dk)
    pool = torch.randn(12, h, dk, dv, generator=torch.Generator().manual_seed(1))
    slots = np.array([3, 11, 0, -1, 7, 12, 5, 2, 1], np.int32)
    state = pool.cuda()
    out = torch.full_like(c.dev("v"), 7.0)
    rows = [c.dev(x) for x in ("q", "k", "v", "g", "beta")]
    o = sla.step_delta(state, torch.from_numpy(slots).cuda(), *rows, out=out)
    ro, rs = delta_ref.delta_step_ref(pool.double().numpy(), slots, *(c.wide(x) for x in ("q", "k", "v", "g", "beta")),
                                      c.scale)
    close(o, ro, dtype, "o")
    close(state, rs, "f32", "state")
    assert (o[[3, 5]] == 7.0).all() and torch.equal(state[[4, 6, 8, 9, 10]].cpu(), pool[[4, 6, 8, 9, 10]])


def test_step_same_slot(sla):
    """Rows of one slot follow each other: a sequence's rows in one call, among other sequences'."""
    import torch

    c = Case([1] * 300, 1, 2, 32, 32, "f32", seed=3)
    slots = np.random.default_rng(2).integers(-1, 5, 300).astype(np.int32)
    pool = torch.randn(5, 2, 32, 32, generator=torch.Generator().manual_seed(1))
    state = pool.cuda()
    o = sla.step_delta(state, torch.from_numpy(slots).cuda(), *(c.dev(x) for x in ("q", "k", "v", "g", "beta")))
    ro, rs = delta_ref.delta_step_ref(pool.double().numpy(), slots, *(c.wide(x) for x in ("q", "k", "v", "g", "beta")),
                                      c.scale)
    close(o, ro, "f32", "o")
    close(state, rs, "f32", "state")


def test_prompt_then_steps(sla):
    """As it is used: a prompt in one call, then row by row on the states it left."""
    import torch

    c = Case([90, 130, 64], 1, 2, 64, 64, "bf16", seed=4)
    whole, last = c.forward(sla)
    rows = [c.dev(x) for x in ("q", "k", "v", "g", "beta")]
    keep = [(0, 80), (90, 210), (220, 280)]
    at = torch.cat([torch.arange(*x) for x in keep]).cuda()
    off = torch.tensor([0, 80, 200, 260], dtype=torch.int32).cuda()
    _, state = sla.forward_delta(*(x[at].contiguous() for x in rows), off)
    slots = torch.arange(3, dtype=torch.int32).cuda()
    for t in range(10):
        now = torch.tensor([80 + t, 210 + t, 280 + t]).cuda()
        live = now < torch.tensor([90, 220, 284]).cuda()
        o = sla.step_delta(state, torch.where(live, slots, -1).to(torch.int32), *(x[now.clamp(max=283)].contiguous() for x in rows))
        ref = whole[now.clamp(max=283)]
        close(o[live], ref[live].double().cpu().numpy(), "bf16", f"o {t}", bar=FP32_BAR + HALF_STEP["bf16"])
    close(state, last.double().cpu().numpy(), "f32", "state")
