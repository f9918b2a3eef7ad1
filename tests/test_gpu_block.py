"""The short convolution, the selective scan and the residual normalisation as a program uses them: one after
the other as a state space block's forward and backward, row by row for answering, in captured graphs, on
several streams, over a plan's windows, and over tensors past 2^31 elements.

Tolerances are those of the operators' own tests, on the inputs each was given; what a whole block gives is held
to sums of those (each operator and product adds its own 1e-5 of the largest value, through gains of a few)."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import space_ref
from tests.gpu_util import torch_dtype
from tests.test_gpu_conv import close

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


class Block:
    """A block of width C: norm, projection to 2 D, convolution, step sizes and maps, scan, projection, norm."""

    def __init__(self, C, D, N, K, dtype, seed=0, device="cuda"):
        import torch

        gen = torch.Generator().manual_seed(seed)
        dt = torch_dtype(dtype)
        rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        R = max(1, C // 8)
        self.C, self.D, self.N, self.R, self.K, self.dt = C, D, N, R, K, dt
        p = dict(w_in=rand(2 * D, C) / C ** 0.5, w_conv=rand(D, K) / K ** 0.5, b_conv=0.1 * rand(D),
                 w_x=rand(R + 2 * N, D) / D ** 0.5, w_dt=rand(D, R) / R ** 0.5, b_dt=-2 + 0.5 * rand(D),
                 A=-(1 + torch.arange(N).float()).expand(D, N) * torch.exp(0.2 * rand(D, N)), skip=1 + 0.1 * rand(D),
                 w_out=rand(C, D) / D ** 0.5, norm=1 + 0.1 * rand(C), next=1 + 0.1 * rand(C))
        self.p = {k: (v.to(dt) if k in ("w_in", "w_x", "w_dt", "w_out") else v).contiguous().to(device) for k, v in p.items()}

    def forward(self, S, x, residual, offsets, conv=None, state=None, keep=False):
        p, D, N, R = self.p, self.D, self.N, self.R
        u, r, rstd, _ = S.forward_residual_norm(x, residual, weight=p["norm"])
        xz = u @ p["w_in"].t()
        c, conv_out = S.forward_short_conv(xz[:, :D], p["w_conv"], offsets, bias=p["b_conv"], activation="silu", state=conv)
        low = c @ p["w_x"].t()
        delta = low[:, :R] @ p["w_dt"].t()
        B, Cm = low[:, R:R + N].unflatten(1, (1, N)), low[:, R + N:].unflatten(1, (1, N))
        y, state_out = S.forward_selective_scan(c, delta, p["A"], B, Cm, offsets, skip=p["skip"], z=xz[:, D:],
                                                delta_bias=p["b_dt"], delta_softplus=True, state=state)
        o = y @ p["w_out"].t()
        out, r2, rstd2, _ = S.forward_residual_norm(o, r, weight=p["next"])
        if not keep:
            return out, r2, conv_out, state_out
        return dict(x=x, u=u, r=r, rstd=rstd, xz=xz, c=c, low=low, delta=delta, B=B, C=Cm, y=y, o=o, out=out, r2=r2, rstd2=rstd2,
                    conv=conv_out, state=state_out)

    def backward(self, S, f, offsets, dout, dr2):
        """Gradients of <out, dout> + <r2, dr2>: of x, the residual rows and every parameter."""
        import torch

        p, D, N, R = self.p, self.D, self.N, self.R
        g = {}
        do, dr, g["next"], _, _ = S.backward_residual_norm(f["o"], f["r2"], dout, f["rstd2"], weight=p["next"],
                                                           dresidual_out=dr2)
        g["w_out"], dy = do.t() @ f["y"], do @ p["w_out"]
        dc, ddelta, g["A"], dB, dC, g["skip"], dz, g["b_dt"], _ = S.backward_selective_scan(
            f["c"], f["delta"], p["A"], f["B"], f["C"], offsets, dy, skip=p["skip"], z=f["xz"][:, D:], delta_bias=p["b_dt"],
            delta_softplus=True)
        g["w_dt"] = ddelta.t() @ f["low"][:, :R]
        dlow = torch.cat([ddelta @ p["w_dt"], dB.flatten(1), dC.flatten(1)], 1)
        g["w_x"], dc = dlow.t() @ f["c"], dc + dlow @ p["w_x"]
        dxc, g["w_conv"], g["b_conv"], _ = S.backward_short_conv(f["xz"][:, :D], p["w_conv"], offsets, dc, bias=p["b_conv"],
                                                                 activation="silu")
        dxz = torch.cat([dxc, dz], 1)
        g["w_in"], du = dxz.t() @ f["u"], dxz @ p["w_in"]
        g["x"], g["residual"], g["norm"], _, _ = S.backward_residual_norm(f["x"], f["r"], du, f["rstd"], weight=p["norm"],
                                                                          dresidual_out=dr)
        return g


def wide_block(b, t, offsets):
    """The block in 64 bits on the CPU, differentiable: (out, r2)."""
    import torch

    p = t
    rms = lambda v: v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
    r = p["residual"] + p["x"]
    xz = (rms(r) * p["norm"]) @ p["w_in"].t()
    D, N, R, K = b.D, b.N, b.R, b.K
    ys = []
    for lo, hi in zip(offsets, offsets[1:]):
        full = torch.cat([torch.zeros(K - 1, D, dtype=torch.float64), xz[lo:hi, :D]])
        c = torch.nn.functional.silu(sum(p["w_conv"][:, j] * full[j:j + hi - lo] for j in range(K)) + p["b_conv"])
        low = c @ p["w_x"].t()
        dt = torch.nn.functional.softplus(low[:, :R] @ p["w_dt"].t() + p["b_dt"])
        h = torch.zeros(D, N, dtype=torch.float64)
        rows = []
        for i in range(hi - lo):
            h = torch.exp(dt[i][:, None] * p["A"]) * h + (dt[i] * c[i])[:, None] * low[i, R:R + N]
            rows.append(h @ low[i, R + N:] + p["skip"] * c[i])
        ys.append(torch.stack(rows) if rows else torch.zeros(0, D, dtype=torch.float64))
    y = torch.cat(ys) * torch.nn.functional.silu(xz[:, D:])
    r2 = r + y @ p["w_out"].t()
    return rms(r2) * p["next"], r2


def test_block_forward_and_backward(sla):
    """A whole block in single precision against 64 bits and its derivative there."""
    import torch

    b = Block(48, 96, 16, 4, "f32", seed=1)
    lengths = [37, 1, 0, 90]
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    offsets = torch.from_numpy(off).cuda()
    gen = torch.Generator().manual_seed(2)
    n = int(off[-1])
    x, residual, dout, dr2 = (torch.randn(n, 48, generator=gen).cuda() for _ in range(4))
    f = b.forward(sla, x, residual, offsets, keep=True)
    g = b.backward(sla, f, offsets, dout, dr2)
    t = {k: v.double().cpu().requires_grad_(True) for k, v in {**b.p, "x": x, "residual": residual}.items()}
    out, r2 = wide_block(b, t, off.tolist())
    ((out * dout.double().cpu()).sum() + (r2 * dr2.double().cpu()).sum()).backward()
    close(f["out"], out.detach().numpy(), "f32", "out", 5e-5)
    close(f["r2"], r2.detach().numpy(), "f32", "r2", 5e-5)
    for k, v in g.items():
        close(v, t[k].grad.numpy(), "f32", k, 1e-4)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_block_operators_on_the_inputs_they_are_given(sla, dtype):
    import torch

    b = Block(64, 128, 16, 4, dtype, seed=3)
    lengths = [70, 3, 55]
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    offsets = torch.from_numpy(off).cuda()
    gen = torch.Generator().manual_seed(4)
    x, residual, dout, dr2 = (torch.randn(128, 64, generator=gen).to(b.dt).cuda() for _ in range(4))
    f = b.forward(sla, x, residual, offsets, keep=True)
    p = {k: num(v) for k, v in b.p.items()}
    ry, rr, _, _ = space_ref.rnorm_forward_ref(num(x), num(residual), p["norm"])
    close(f["u"], ry, dtype, "u")
    close(f["r"], rr, dtype, "r")
    rc, _ = space_ref.conv_forward_ref(num(f["xz"][:, :128]), p["w_conv"], off, p["b_conv"], "silu")
    close(f["c"], rc, dtype, "c")
    ry, rs = space_ref.scan_forward_ref(num(f["c"]), num(f["delta"]), p["A"], num(f["B"]), num(f["C"]), off, p["skip"],
                                        num(f["xz"][:, 128:]), p["b_dt"], True)
    close(f["y"], ry, dtype, "y")
    close(f["state"], rs, "f32", "state")
    g = b.backward(sla, f, offsets, dout, dr2)
    assert all(torch.isfinite(v).all() for v in g.values())


def test_answering_row_by_row(sla):
    """A prompt at once, then rows one by one on pools of states, for several sequences in turn: what all rows at
    once give, to sums of the operators' tolerances."""
    import torch

    b = Block(32, 64, 16, 4, "f32", seed=5)
    gen = torch.Generator().manual_seed(6)
    n, prompt = 30, 21
    seqs = [(torch.randn(n, 32, generator=gen).cuda(), torch.randn(n, 32, generator=gen).cuda()) for _ in range(3)]
    cat = lambda xs: torch.cat(xs)  # noqa: E731
    whole, _, conv_end, state_end = b.forward(sla, cat([s[0] for s in seqs]), cat([s[1] for s in seqs]),
                                              torch.tensor([0, n, 2 * n, 3 * n], dtype=torch.int32).cuda())
    out, _, conv, state = b.forward(sla, cat([s[0][:prompt] for s in seqs]), cat([s[1][:prompt] for s in seqs]),
                                    torch.tensor([0, prompt, 2 * prompt, 3 * prompt], dtype=torch.int32).cuda())
    # the pools have a place more, in another order
    place = [3, 0, 2]
    convs, states = torch.zeros(4, 3, 64).cuda(), torch.zeros(4, 64, 16).cuda()
    for i, s in enumerate(place):
        convs[s], states[s] = conv[i], state[i]
    slots = torch.tensor(place, dtype=torch.int32).cuda()
    p = b.p
    for t in range(prompt, n):
        x, r = cat([s[0][t:t + 1] for s in seqs]), cat([s[1][t:t + 1] for s in seqs])
        u, r, _, _ = sla.forward_residual_norm(x, r, weight=p["norm"])
        xz = u @ p["w_in"].t()
        c = sla.step_short_conv(convs, slots, xz[:, :64], p["w_conv"], p["b_conv"], "silu")
        low = c @ p["w_x"].t()
        y = sla.step_selective_scan(states, slots, c, low[:, :b.R] @ p["w_dt"].t(), p["A"],
                                    low[:, b.R:b.R + 16].unflatten(1, (1, 16)), low[:, b.R + 16:].unflatten(1, (1, 16)),
                                    skip=p["skip"], z=xz[:, 64:], delta_bias=p["b_dt"], delta_softplus=True)
        got, _, _, _ = sla.forward_residual_norm(y @ p["w_out"].t(), r, weight=p["next"])
        want = whole.view(3, n, 32)[:, t]
        assert (got - want).abs().max() <= 5e-5 * whole.abs().max(), t
    assert (convs[place] - conv_end).abs().max() <= 2e-5 * conv_end.abs().max()
    assert (states[place] - state_end).abs().max() <= 5e-5 * state_end.abs().max()
    assert (states[1] == 0).all() and (convs[1] == 0).all()


def calls(S, t, off, ws=None, outs=None):
    """Every operator once, forward and backward, and the single rows: [outputs]."""
    ws, o = ws or {}, outs or {}
    kw = dict(skip=t["skip"], z=t["z"], delta_bias=t["bias"], delta_softplus=True)
    rows = (t["x"], t["delta"], t["A"], t["B"], t["C"])
    y, fin = S.forward_short_conv(t["x"], t["w"], off, bias=t["bias"], activation="silu", y=o.get("y"),
                                  final_state=o.get("fin"))
    dx, dw, db, _ = S.backward_short_conv(t["x"], t["w"], off, t["dy"], bias=t["bias"], activation="silu",
                                          workspace=ws.get("conv"), dx=o.get("dx"))
    s, st = S.forward_selective_scan(*rows, off, workspace=ws.get("scan"), y=o.get("s"), final_state=o.get("st"), **kw)
    g = S.backward_selective_scan(*rows, off, t["dy"], workspace=ws.get("back"), out=o.get("g"), **kw)
    n, r, rstd, ps = S.forward_residual_norm(s, t["r"], weight=t["skip"], post_weight=t["bias"], gate=t["z"],
                                             activation="silu", y=o.get("n"), residual_out=o.get("ro"))
    h = S.backward_residual_norm(s, r, t["dy"], rstd, weight=t["skip"], post_weight=t["bias"], post_rstd=ps, gate=t["z"],
                                 activation="silu", workspace=ws.get("norm"), dx=o.get("dn"), dresidual=o.get("dr"))
    return [v for v in (y, fin, dx, dw, db, s, st, *g, n, r, rstd, ps, *h) if v is not None]


def inputs(dtype, lengths, D=72, N=16, seed=0):
    import torch

    gen = torch.Generator().manual_seed(seed)
    dt, n = torch_dtype(dtype), sum(lengths)
    rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    t = dict(x=rand(n, D).to(dt), delta=(0.3 * rand(n, D)).to(dt), B=rand(n, 1, N).to(dt), C=rand(n, 1, N).to(dt),
             z=rand(n, D).to(dt), dy=rand(n, D).to(dt), r=rand(n, D), A=-1 - 4 * torch.rand(D, N, generator=gen), skip=rand(D),
             bias=rand(D) - 1, w=rand(D, 4))
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
    return {k: v.cuda() for k, v in t.items()}, off


def workspaces(S, n, W, dt, D, N):
    import torch

    new = lambda b: torch.empty(b, dtype=torch.uint8, device="cuda")  # noqa: E731
    return dict(conv=new(S.short_conv_backward_workspace_bytes(n, W, dt, D, 4)),
                scan=new(S.selective_scan_workspace_bytes(n, W, dt, D, 1, N)),
                back=new(S.selective_scan_backward_workspace_bytes(n, W, dt, D, 1, N)),
                norm=new(S.residual_norm_backward_workspace_bytes(n, dt, D)))


@pytest.mark.parametrize("lengths,dtype", [([130, 1, 0, 64, 77], "bf16"), ([900, 300], "f32")])
def test_operators_in_a_graph(sla, lengths, dtype):
    """All calls captured, replayed on new inputs with eager work between the replays: each replay is the eager
    result, and a second graph that shares the workspaces, replayed after it, too."""
    import torch

    t, off = inputs(dtype, lengths)
    n, W, D, N = sum(lengths), len(lengths), 72, 16
    ws = workspaces(sla, n, W, t["x"].dtype, D, N)
    pool_c, pool_s = torch.zeros(4, 3, D, dtype=t["x"].dtype).cuda(), torch.zeros(4, D, N).cuda()
    slots = torch.tensor([2, 0, 2, -1], dtype=torch.int32).cuda()

    def steps(pool_c, pool_s):
        c = sla.step_short_conv(pool_c, slots, t["x"][:4], t["w"], t["bias"], "silu", y=torch.zeros_like(t["x"][:4]))
        s = sla.step_selective_scan(pool_s, slots, t["x"][:4], t["delta"][:4], t["A"], t["B"][:4], t["C"][:4], skip=t["skip"],
                                    z=t["z"][:4], delta_bias=t["bias"], delta_softplus=True, y=torch.zeros_like(t["x"][:4]))
        return [c, s]

    calls(sla, t, off, ws)
    steps(pool_c, pool_s)
    torch.cuda.synchronize()
    graphs, got = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(calls(sla, t, off, ws) + steps(pool_c, pool_s))
        graphs.append(g)
    for r in range(4):
        new, _ = inputs(dtype, lengths, seed=10 + r)
        for k, v in new.items():
            t[k].copy_(v)
        for which in (0, 1):
            pool_c.fill_(0.5 * r)
            pool_s.fill_(0.25 * r)
            mine = pool_c.clone(), pool_s.clone()
            want = calls(sla, t, off) + steps(*mine)
            graphs[which].replay()
            torch.cuda.synchronize()
            for a, b in zip(got[which], want):
                assert torch.equal(a, b)
            assert torch.equal(pool_c, mine[0]) and torch.equal(pool_s, mine[1])


def test_two_streams(sla):
    import torch

    lengths = [900, 300, 64]
    want = []
    for i in range(2):
        t, off = inputs("bf16", lengths, seed=i)
        want.append((t, off, calls(sla, t, off)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, (t, off, _) in zip(streams, want):
            with torch.cuda.stream(s):
                got.append(calls(sla, {k: v.clone() for k, v in t.items()}, off))
        torch.cuda.synchronize()
        for g, (_, _, w) in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_over_a_plan_behind_attention(sla):
    """The windows and row order of an attention's plan: the convolution and the scan take them as they are."""
    import torch

    gen = torch.Generator().manual_seed(1)
    n, W, H, d = 1200, 40, 4, 32
    win = torch.randint(0, W, (n,), generator=gen).to(torch.int32).cuda()
    plan = sla.build_segments(win, num_windows=W)
    q, k, v = (torch.randn(n, H, d, generator=gen).cuda() for _ in range(3))
    x = sla.forward(plan, q, k, v).reshape(n, H * d)
    w = torch.randn(H * d, 3, generator=gen).cuda()
    _, perm, offs, _, _ = sla.read_plan(plan)
    y, st = sla.forward_short_conv(x, w, plan.offsets, activation="silu", order=plan.perm)
    ry, rs = space_ref.conv_forward_ref(num(x), num(w), offs, activation="silu", order=perm)
    close(y, ry, "f32", "y")
    assert (num(st) == rs).all()
    A = -torch.rand(H * d, 8, generator=gen).cuda() - 0.5
    B, C = (torch.randn(n, 2, 8, generator=gen).cuda() for _ in range(2))
    delta = torch.rand(n, H * d, generator=gen).cuda()
    s, h = sla.forward_selective_scan(y, delta, A, B, C, plan.offsets, order=plan.perm)
    rs, rh = space_ref.scan_forward_ref(num(y), num(delta), num(A), num(B), num(C), offs, order=perm)
    close(s, rs, "f32", "scan")
    close(h, rh, "f32", "state")


def test_rows_past_two_billion_elements(sla):
    """Rows of more than 2^31 elements: the last windows are what they are alone."""
    import torch

    lengths = [1000] * 525 + [300, 37]
    n, D, N = sum(lengths), 4096, 4
    assert n * D > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(0)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    x, delta, dy = new(n, D), new(n, D), new(n, D)
    B, C = new(n, 1, N), new(n, 1, N)
    A, w = -1 - torch.rand(D, N, device="cuda", generator=gen), torch.randn(D, 4, device="cuda", generator=gen)
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
    last = torch.tensor([0, 300, 337], dtype=torch.int32).cuda()
    tail = [t[-337:].clone() for t in (x, delta, dy, B, C)]
    y, st = sla.forward_short_conv(x, w, off, activation="silu")
    y2, st2 = sla.forward_short_conv(tail[0], w, last, activation="silu")
    assert torch.equal(y[-337:], y2) and torch.equal(st[-2:], st2)
    dx, _, _, _ = sla.backward_short_conv(x, w, off, dy, activation="silu", dx=y)
    dx2, _, _, _ = sla.backward_short_conv(tail[0], w, last, tail[2], activation="silu")
    assert torch.equal(dx[-337:], dx2)
    y, st = sla.forward_selective_scan(x, delta, A, B, C, off, delta_softplus=True, y=y)
    y2, st2 = sla.forward_selective_scan(tail[0], tail[1], A, tail[3], tail[4], last, delta_softplus=True)
    # the cut of a window depends on how many rows there are in all
    assert (y[-337:].float() - y2.float()).abs().max() <= 2.0 ** -7 * y2.float().abs().max()
    assert (st[-2:] - st2).abs().max() <= 2e-5 * st2.abs().max()
    n1, r1, _, _ = sla.forward_residual_norm(x, delta, activation="silu", gate=dy, y=y)
    n2, r2, _, _ = sla.forward_residual_norm(tail[0], tail[1], activation="silu", gate=tail[2])
    assert torch.equal(n1[-337:], n2) and torch.equal(r1[-337:], r2)
    del n1, r1, y, dx
    g = sla.backward_selective_scan(x, delta, A, B, C, off, dy, delta_softplus=True)
    g2 = sla.backward_selective_scan(tail[0], tail[1], A, tail[3], tail[4], last, tail[2], delta_softplus=True)
    for i in (0, 1, 3, 4):
        assert (g[i][-337:].float() - g2[i].float()).abs().max() <= 2.0 ** -7 * g2[i].float().abs().max()


def test_states_past_two_billion_elements(sla):
    import torch

    slots, D, N = 17000, 8192, 16
    assert slots * D * N > 2 ** 31
    pool = torch.empty(slots, D, N, device="cuda")
    gen = torch.Generator().manual_seed(2)
    use = [slots - 1, 0, 16500]
    small = torch.randn(3, D, N, generator=gen).cuda()
    for i, s in enumerate(use):
        pool[s] = small[i]
    t, _ = inputs("bf16", [3], D=D, N=N)
    args = [t[k] for k in ("x", "delta", "A", "B", "C")]
    y = sla.step_selective_scan(pool, torch.tensor(use, dtype=torch.int32).cuda(), *args, delta_softplus=True)
    y2 = sla.step_selective_scan(small, torch.arange(3, dtype=torch.int32).cuda(), *args, delta_softplus=True)
    assert torch.equal(y, y2) and all(torch.equal(pool[s], small[i]) for i, s in enumerate(use))


def test_same_results_twice(sla):
    """No sum's order changes from call to call."""
    import torch

    for dtype in ("bf16", "f32"):
        t, off = inputs(dtype, [700, 0, 33, 1, 260], D=200, N=24, seed=9)
        a = calls(sla, t, off)
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(a, calls(sla, t, off)))
