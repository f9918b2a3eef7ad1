"""The selective scan, its gradients and its single rows against the float64 reference.

Tolerances.  A decay exp(x) is off by |x| 2^-23 of itself, and each row adds two roundings (2^-23 in all) to
what a state holds; what a row wrote k rows ago weighs e^-(k a) for a rate a of forgetting, so its error
is at most (k a + k) 2^-23 e^-(k a) <= (1 + 1 / a) 2^-23 / e of the largest it has been: 9e-7 for a = 0.05,
the slowest rate of these inputs (step sizes above 0.05 at A = -1).  A sum of 64 states adds 64 * 2^-24 of
its terms in the worst case.  1e-5 of the largest result covers them.  Where nothing is forgotten over m rows, the
bound is m 2^-23, and the tests that have that say so.  A 16-bit result is off by half a step of its value more.
A parameter's gradient is a sum over all rows: its limit is 1e-5 of the sum of its terms' sizes, which the
reference gives for the same rows without their signs."""
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
ROWS = ("x", "delta", "A", "B", "C")
OPTIONS = ("skip", "z", "delta_bias")
GRADS = ("dx", "ddelta", "dA", "dB", "dC", "dskip", "dz", "ddelta_bias", "dstate_in")


class Case:
    def __init__(self, lengths, D, N, dtype, G=1, seed=0, skip=True, gate=True, bias=True, softplus=True, state=False,
                 order=False, front=0, behind=0, strided=False, slow=False):
        import torch

        gen = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        uniform = lambda lo, hi, *s: lo + (hi - lo) * torch.rand(*s, generator=gen)  # noqa: E731
        n = self.n = front + sum(lengths) + behind
        self.w, self.D, self.N, self.G, self.dtype = len(lengths), D, N, G, dtype
        dt = torch_dtype(dtype)
        self.offsets = (front + np.concatenate([[0], np.cumsum(lengths)])).astype(np.int32)
        self.off = torch.from_numpy(self.offsets).cuda()

        def rows(*shape, scale=1.0):
            t = (scale * normal(n, *shape)).to(dt)
            if not strided:
                return t.cuda()
            wide = torch.full((n, 3 + t[0].numel() + 4 if n else 7), 9.0, dtype=dt)
            wide[:, 3:-4] = t.reshape(n, -1)
            return wide.cuda()[:, 3:-4].unflatten(1, shape) if len(shape) > 1 else wide.cuda()[:, 3:-4]

        r = dict(x=rows(D), delta=rows(D, scale=0.3), B=rows(G, N), C=rows(G, N), dy=rows(D), z=rows(D) if gate else None)
        r["A"] = (-uniform(0.0, 0.001, D, N) if slow else -uniform(1.0, 8.0, D, N)).cuda()
        r["delta_bias"] = uniform(-2.0, -1.0, D).cuda() if bias else None
        if not softplus:
            r["delta"] = (r["delta"].abs() + 0.06)
            r["delta_bias"] = None if r["delta_bias"] is None else uniform(0.0, 0.2, D).cuda()
        r["skip"] = normal(D).cuda() if skip else None
        self.state = normal(self.w, D, N).cuda() if state else None
        self.dstate = normal(self.w, D, N).cuda() if state else None
        self.order = torch.randperm(n, generator=gen).to(torch.int32).cuda() if order else None
        self.r = r
        self.kw = dict({k: r[k] for k in OPTIONS}, delta_softplus=softplus, order=self.order, state=self.state)
        self.ref_kw = dict({k: num(r[k]) for k in OPTIONS}, delta_softplus=softplus, state=num(self.state),
                           order=None if self.order is None else self.order.cpu().numpy())
        self.new = lambda t: torch.full(t.shape, 7.0, dtype=t.dtype).cuda()

    def args(self):
        return [self.r[k] for k in ROWS]

    def forward(self, S, bar=1e-5):
        y, st = S.forward_selective_scan(*self.args(), self.off, y=self.new(self.r["x"]), **self.kw)
        ry, rs = space_ref.scan_forward_ref(*map(num, self.args()), self.offsets, **self.ref_kw)
        close(y, ry, self.dtype, "y", bar)
        close(st, rs, "f32", "state", bar)
        return y, st

    def gradients(self, S, **more):
        outs = [self.new(self.r[k]) for k in ("x", "delta", "B", "C")] + [None if self.r["z"] is None else self.new(self.r["z"])]
        return S.backward_selective_scan(*self.args(), self.off, self.r["dy"], dstate=self.dstate, out=outs, **self.kw,
                                         **more)

    def backward(self, S, bar=1e-5):
        got = dict(zip(GRADS, self.gradients(S)))
        ref_args = (*map(num, self.args()), self.offsets, num(self.r["dy"]))
        ref = dict(zip(GRADS, space_ref.scan_backward_ref(*ref_args, dstate=num(self.dstate), **self.ref_kw)))
        for name, given in (("dskip", "skip"), ("dz", "z"), ("ddelta_bias", "delta_bias")):
            assert (got[name] is None) == (self.r[given] is None), name
        assert (got["dstate_in"] is None) == (self.state is None)
        for name in ("dx", "ddelta", "dB", "dC", "dz"):
            if got[name] is not None:
                close(got[name], ref[name], self.dtype, name, bar)
        if self.state is not None:
            close(got["dstate_in"], ref["dstate_in"], "f32", "dstate_in", bar)
        # the sizes of the parameters' terms: every factor without its sign
        size = {k: None if v is None else np.abs(v) for k, v in dict(zip(ROWS, ref_args[:5])).items()}
        size["A"] = ref_args[2]
        kw = dict(self.ref_kw, state=None if self.state is None else np.abs(num(self.state)))
        dt = ref_args[1] if kw["delta_bias"] is None else ref_args[1] + kw["delta_bias"]
        kw.update(delta_softplus=False, delta_bias=None, z=None,
                  skip=None if kw["skip"] is None else np.abs(kw["skip"]))
        size["delta"] = np.logaddexp(0, dt) if self.kw["delta_softplus"] else dt
        dy = np.abs(ref_args[6])
        if self.ref_kw["z"] is not None:
            dy = dy * np.abs(space_ref._act("silu", self.ref_kw["z"]))
        most = dict(zip(GRADS, space_ref.scan_backward_ref(*(size[k] for k in ROWS), self.offsets, dy,
                                                           dstate=None if self.dstate is None else np.abs(num(self.dstate)),
                                                           **kw)))
        within(got["dA"], ref["dA"], bar * most["dA"], "dA")
        if got["dskip"] is not None:
            within(got["dskip"], ref["dskip"], bar * most["dskip"], "dskip")
        if got["ddelta_bias"] is not None:
            # without signs, |du x| + |da A|: A's part is negative in `most`
            flip = dict(zip(GRADS, space_ref.scan_backward_ref(*(size[k] if k != "A" else 0 * size[k] for k in ROWS),
                                                               self.offsets, dy, dstate=None, **dict(kw, state=None))))
            limit = bar * (np.abs(most["dA"] * size["A"]).sum(-1) / 0.05 + flip["ddelta_bias"])
            within(got["ddelta_bias"], ref["ddelta_bias"], limit + bar * np.abs(ref["ddelta_bias"]).max(), "ddelta_bias")
        return got


SHAPES = [(1, 1, 1), (3, 2, 1), (64, 4, 1), (70, 5, 1), (64, 8, 1), (130, 16, 1), (48, 12, 3), (256, 16, 2), (20, 24, 1),
          (65, 32, 1), (36, 64, 2), (100, 33, 4), (12, 3, 12)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,N,G", SHAPES)
def test_forward_shapes(sla, dtype, D, N, G):
    Case([5, 0, 1, 70, 33, 2, 0, 140], D, N, dtype, G, seed=D + N, state=N % 2 == 0, front=2, behind=3).forward(sla)


LENGTHS = [[1], [0], [2], [7, 8, 9], [16], [17], [63, 64, 65], [128], [129], [0, 0, 1], [1] * 70, [300], [64, 0, 192, 1, 640]]


@pytest.mark.parametrize("lengths", LENGTHS)
def test_forward_lengths(sla, lengths):
    for state in (False, True):
        Case(lengths, 40, 16, "f32", seed=3, state=state).forward(sla)
        Case(lengths, 9, 6, "bf16", 3, seed=4, state=state, behind=1).forward(sla)


@pytest.mark.parametrize("kw", [dict(skip=False), dict(gate=False), dict(bias=False), dict(softplus=False),
                                dict(skip=False, gate=False, bias=False, softplus=False)])
def test_forward_options(sla, kw):
    Case([40, 90, 3], 80, 16, "f32", seed=5, state=True, **kw).forward(sla)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_and_order(sla, dtype):
    for kw in (dict(strided=True), dict(order=True), dict(order=True, strided=True)):
        Case([30, 4, 150], 96, 16, dtype, 2, seed=6, state=True, behind=2, front=1, **kw).forward(sla)


def test_forward_of_long_windows_that_forget_nothing(sla):
    """Parts of a window hand on all they hold: 3,000 rows' roundings, two each."""
    c = Case([3000, 700], 24, 16, "f32", seed=7, state=True, slow=True)
    c.forward(sla, bar=3700 * 2.0 ** -23)
    c = Case([9000], 16, 4, "bf16", seed=8)
    c.forward(sla)


def test_state_in_place(sla):
    import torch

    for lengths in ([40, 0, 3], [700, 64, 65, 0, 1300]):
        c = Case(lengths, 72, 16, "f32", seed=9, state=True)
        y, st = c.forward(sla)
        for _ in range(3):
            pool = c.state.clone()
            y2, _ = sla.forward_selective_scan(*c.args(), c.off, y=c.new(y), final_state=pool, **{**c.kw, "state": pool})
            assert torch.equal(y, y2) and torch.equal(st, pool)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,N,G", [(1, 1, 1), (7, 3, 1), (64, 8, 2), (300, 16, 1), (90, 12, 3), (48, 32, 1), (40, 64, 1),
                                   (1030, 5, 1)])
def test_single_rows(sla, dtype, D, N, G):
    import torch

    slots = torch.tensor([3, 0, 3, -1, 5, 3, 7, 0], dtype=torch.int32)
    for kw in (dict(), dict(strided=True), dict(gate=False, skip=False)):
        c = Case([8], D, N, dtype, G, seed=D, **kw)
        pool = torch.randn(7, D, N, generator=torch.Generator().manual_seed(1)).cuda()
        opts = {k: c.r[k] for k in OPTIONS}
        ry, rs = space_ref.scan_step_ref(num(pool), slots.numpy(), *map(num, c.args()), **{k: num(v) for k, v in opts.items()},
                                         delta_softplus=True)
        y = sla.step_selective_scan(pool, slots.cuda(), *c.args(), **opts, delta_softplus=True, y=c.new(c.r["x"]))
        close(y, ry, dtype, "y")
        close(pool, rs, "f32", "state")


def test_steps_are_the_forward(sla):
    import torch

    c = Case([150], 72, 16, "f32", seed=12, state=True)
    y, st = c.forward(sla)
    pool, slot = c.state.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    opts = dict(skip=c.r["skip"], delta_bias=c.r["delta_bias"], delta_softplus=True)
    got = torch.cat([sla.step_selective_scan(pool, slot, *(c.r[k] if k == "A" else c.r[k][t:t + 1] for k in ROWS),
                                             z=c.r["z"][t:t + 1], **opts) for t in range(150)])
    # both are within 1e-5 of the reference's largest
    assert (got - y).abs().max() <= 2e-5 * y.abs().max() and (pool - st).abs().max() <= 2e-5 * st.abs().max()


def test_extreme_step_sizes(sla):
    """Steps that forget everything, that are 0, and softplus far from 0 on both sides."""
    import torch

    c = Case([70, 10], 64, 16, "f32", seed=13, state=True, bias=False)
    c.r["delta"][3] = 1000.0
    c.r["delta"][5] = -1000.0
    c.r["delta"][6] = -30.0
    c.r["delta"][65] = 60.0
    c.forward(sla)
    c = Case([200], 64, 16, "f32", seed=14, state=True, softplus=False, bias=False)
    c.r["delta"][10:20] = 0.0
    c.r["A"][3] = -float("inf")
    c.r["delta"][:, 3] = c.r["delta"][:, 3].abs() + 0.1
    c.forward(sla)
    # a state that grows, but whose values stay finite: exp of a part's sum of steps alone would not
    c = Case([600], 64, 4, "f32", seed=15, state=True, softplus=False, bias=False, gate=False)
    c.r["A"][:] = 1.0
    c.r["delta"][:] = 0.25
    c.state[:] = 1e-30
    c.r["x"][:] = 0.0
    c.kw["state"], c.ref_kw["state"] = c.state, num(c.state)
    # the growth's exponent, 150, is off by 150 2^-23 in a product of 600 factors off by 2^-23 each
    c.forward(sla, bar=1e-4)


def test_values_that_are_not_finite_stay_in_their_window_and_channel(sla):
    import torch

    c = Case([100, 100], 70, 16, "f32", seed=16)
    c.r["x"][20, 3], c.r["z"][30, 5] = float("nan"), float("inf")
    y, st = sla.forward_selective_scan(*c.args(), c.off, **c.kw)
    want = torch.zeros_like(y, dtype=torch.bool)
    want[20:100, 3] = True
    want[30, 5] = True
    assert torch.equal(~torch.isfinite(y), want)
    bad = torch.zeros(2, 70, dtype=torch.bool, device="cuda")
    bad[0, 3] = True
    assert torch.equal((~torch.isfinite(st)).any(-1), bad)


WRONG = ([0, 200, 100, 300, 250, 700], [-5, 300, 900, 10, 10, 2000], [700, 600, 500, 400, 0, 700], [0, 2000, 0, 2000, 0, 2000])


@pytest.mark.parametrize("fill", [0, 0x7f, 0xff])
@pytest.mark.parametrize("offsets", WRONG)
def test_wrong_offsets_stay_in_range(sla, offsets, fill):
    import torch

    n, D, N = 700, 40, 8
    c = Case([n], D, N, "bf16", seed=17)
    off = torch.tensor(offsets, dtype=torch.int32).cuda()
    w = len(offsets) - 1
    state = torch.randn(w, D, N).cuda()
    bad = torch.arange(n, dtype=torch.int32).cuda() * 3 - n
    for order in (None, bad):
        y, fin = torch.full((3, n, D), 7.0, dtype=c.r["x"].dtype).cuda(), torch.full((3, w, D, N), 7.0).cuda()
        ws = torch.full((sla.selective_scan_workspace_bytes(n, w, y.dtype, D, 1, N),), fill, dtype=torch.uint8).cuda()
        sla.forward_selective_scan(*c.args(), off, y=y[1], final_state=fin[1], workspace=ws,
                                   **{**c.kw, "order": order, "state": state})
        torch.cuda.synchronize()
        for t in (y, fin):
            assert (t[0] == 7.0).all() and (t[2] == 7.0).all()


# ------------------------------------------------------------------ gradients
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,N,G", SHAPES)
def test_backward_shapes(sla, dtype, D, N, G):
    Case([5, 0, 1, 70, 33, 2, 0, 140], D, N, dtype, G, seed=D + N, state=N % 2 == 0, front=2, behind=3).backward(sla)


@pytest.mark.parametrize("lengths", LENGTHS)
def test_backward_lengths(sla, lengths):
    for state in (False, True):
        Case(lengths, 40, 16, "f32", seed=3, state=state).backward(sla)
        Case(lengths, 9, 6, "bf16", 3, seed=4, state=state, behind=1).backward(sla)


@pytest.mark.parametrize("kw", [dict(skip=False), dict(gate=False), dict(bias=False), dict(softplus=False),
                                dict(skip=False, gate=False, bias=False, softplus=False)])
def test_backward_options(sla, kw):
    Case([40, 90, 3], 80, 16, "f32", seed=5, state=True, **kw).backward(sla)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_strided_rows_and_order(sla, dtype):
    for kw in (dict(strided=True), dict(order=True), dict(order=True, strided=True)):
        Case([30, 4, 150], 96, 16, dtype, 2, seed=6, state=True, behind=2, front=1, **kw).backward(sla)


def test_backward_of_long_windows(sla):
    """Many parts; where nothing is forgotten, all of 2,300 rows' roundings stay."""
    Case([1800, 500], 24, 16, "f32", seed=7, state=True).backward(sla)
    Case([1800, 500], 24, 16, "f32", seed=7, state=True, slow=True).backward(sla, bar=2300 * 2.0 ** -23)
    Case([3000], 300, 4, "bf16", seed=8).backward(sla)


def test_gradients_by_differences(sla):
    import torch

    c = Case([30, 3, 41], 12, 5, "f32", 2, seed=18, state=True)
    got = dict(zip(GRADS, c.gradients(sla)))
    rows = {k: c.r[k] for k in (*ROWS, *OPTIONS)}
    rows["state"] = c.state

    def loss(r):
        host = {k: num(v) for k, v in r.items()}
        y, st = space_ref.scan_forward_ref(*(host[k] for k in ROWS), c.offsets, *(host[k] for k in OPTIONS),
                                           delta_softplus=True, state=host["state"])
        return (y * num(c.r["dy"])).sum() + (st * num(c.dstate)).sum()

    gen = torch.Generator().manual_seed(1)
    for name, grad in (("x", "dx"), ("delta", "ddelta"), ("A", "dA"), ("B", "dB"), ("C", "dC"), ("skip", "dskip"),
                       ("z", "dz"), ("delta_bias", "ddelta_bias"), ("state", "dstate_in")):
        d = torch.randn(rows[name].shape, generator=gen, dtype=torch.float64)
        up, down = (loss({**rows, name: rows[name].double().cpu() + s * 1e-4 * d}) for s in (1, -1))
        mine = float((got[grad].double().cpu() * d).sum())
        # the difference's own error is 1e-8 of a third derivative; the gradient's 1e-5 of its size
        assert abs((up - down) / 2e-4 - mine) <= 1e-5 * float(got[grad].double().norm() * d.norm()) + 1e-6, name


def test_gradient_of_the_state_in_place(sla):
    """dstate_in where dstate_out lies: the first part's workgroup writes what the last one's reads."""
    import torch

    for lengths in ([40, 0, 3], [700, 64, 33, 0, 400]):
        c = Case(lengths, 72, 16, "f32", seed=19, state=True)
        want = c.gradients(sla)
        n, w = c.n, c.w
        for _ in range(3):
            ds = c.dstate.clone()
            outs = [torch.zeros_like(c.r[k]) for k in ("x", "delta")]
            par = [torch.zeros_like(c.r["A"]), torch.zeros_like(c.r["B"]), torch.zeros_like(c.r["C"]),
                   torch.zeros_like(c.r["skip"]), torch.zeros_like(c.r["z"]), torch.zeros_like(c.r["skip"])]
            need = sla.selective_scan_backward_workspace_bytes(n, w, torch.float32, 72, 1, 16)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            p = lambda t: t.data_ptr()  # noqa: E731
            r = c.r
            rc = sla.lib().sla_backward_selective_scan(
                p(c.off), n, w, None, 0, 72, 1, 16, 1, p(r["x"]), 72, p(r["delta"]), 72, p(r["A"]), p(r["B"]), 16, p(r["C"]),
                16, p(r["skip"]), p(r["z"]), 72, p(r["delta_bias"]), p(c.state), p(r["dy"]), 72, p(ds), *map(p, outs),
                *map(p, par), p(ds), p(ws), need, torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            for a, b in zip((*outs, *par, ds), want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("fill", [0, 0x7f, 0xff])
@pytest.mark.parametrize("offsets", WRONG)
def test_backward_wrong_offsets_stay_in_range(sla, offsets, fill):
    import torch

    n, D, N = 700, 40, 8
    c = Case([n], D, N, "bf16", seed=17)
    off = torch.tensor(offsets, dtype=torch.int32).cuda()
    w = len(offsets) - 1
    state = torch.randn(w, D, N).cuda()
    bad = torch.arange(n, dtype=torch.int32).cuda() * 3 - n
    for order in (None, bad):
        ws = torch.full((sla.selective_scan_backward_workspace_bytes(n, w, torch.bfloat16, D, 1, N),), fill,
                        dtype=torch.uint8).cuda()
        outs = [torch.full((3, *c.r[k].shape), 7.0, dtype=torch.bfloat16).cuda() for k in ("x", "delta", "B", "C", "z")]
        sla.backward_selective_scan(*c.args(), off, c.r["dy"], dstate=state, out=[t[1] for t in outs], workspace=ws,
                                    **{**c.kw, "order": order, "state": state})
        torch.cuda.synchronize()
        for t in outs:
            assert (t[0] == 7.0).all() and (t[2] == 7.0).all()


def test_workspace_contents_do_not_matter(sla):
    import torch

    for lengths, N in (([130, 1, 0, 64, 7], 16), ([700, 300], 5)):
        c = Case(lengths, 72, N, "f32", seed=20, behind=5, order=True, state=True)
        got = []
        for fill in (0, 0xff, 0x7b):
            size = (c.n, c.w, torch.float32, 72, 1, N)
            ws = torch.full((max(sla.selective_scan_backward_workspace_bytes(*size),
                                 sla.selective_scan_workspace_bytes(*size)),), fill, dtype=torch.uint8).cuda()
            y, st = sla.forward_selective_scan(*c.args(), c.off, y=c.new(c.r["x"]), workspace=ws, **c.kw)
            ws.fill_(fill)
            got.append([y, st, *c.gradients(sla, workspace=ws)])
        for g in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got[0], g))


def test_parameters_and_states_at_any_address(sla):
    import torch

    c = Case([70, 30], 72, 16, "f32", seed=21, state=True)
    odd = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
    a = [*c.forward(sla), *c.gradients(sla)]
    slots = torch.tensor([1, 0], dtype=torch.int32).cuda()
    row = {k: c.r[k][:2] for k in ("x", "delta", "B", "C", "z")}
    step = lambda pool, A, skip: sla.step_selective_scan(  # noqa: E731
        pool, slots, row["x"], row["delta"], A, row["B"], row["C"], skip=skip, z=row["z"], delta_softplus=True)
    pool, other = c.state.clone(), odd(c.state)
    y = step(pool, c.r["A"], c.r["skip"])
    for k in ("A", "skip", "delta_bias"):
        c.r[k] = odd(c.r[k])
    c.kw.update(skip=c.r["skip"], delta_bias=c.r["delta_bias"], state=odd(c.state))
    c.dstate = odd(c.dstate)
    b = [*c.forward(sla), *c.gradients(sla)]
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert torch.equal(y, step(other, c.r["A"], c.r["skip"])) and torch.equal(pool, other)


def test_an_infinite_gradient_stays_in_its_row_and_window(sla):
    """dy of one row: its own gradients, and those of the rows before it in its window and channel (its group's
    for B and C), are not finite; no others are."""
    import torch

    c = Case([40, 50], 32, 8, "f32", 2, seed=22, state=True)
    c.r["dy"][60, 20] = float("inf")
    got = dict(zip(GRADS, c.gradients(sla)))
    for name in ("dx", "ddelta", "dz"):
        bad = ~torch.isfinite(got[name])
        assert bad[60, 20] and not bad[:40].any() and not bad[61:].any(), name
        bad[:, 20] = False
        assert not bad.any(), name
    for name in ("dB", "dC"):
        bad = ~torch.isfinite(got[name])
        assert not bad[:, 0].any() and not bad[:40].any() and not bad[61:].any(), name
    assert torch.isfinite(got["dstate_in"][0]).all()
    assert torch.isfinite(got["dA"][:16]).all() and torch.isfinite(got["dskip"][:16]).all()
