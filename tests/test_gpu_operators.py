"""The gated delta rule and group normalisation as a program uses them: one after the other as a
layer's forward and backward, behind the attention, in captured graphs, on several streams, on
workspaces that held something else, over tensors past 2^31 elements, and on offsets that are
wrong.

Tolerances are those of the operators' own tests: 1e-5 of the largest result for fp32, half a step
of the value more for 16 bits; where a 16-bit result is the next operator's input, that rounding
(2^-8 or 2^-11 of a value) reaches the next result once more."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import delta_ref
from tests.test_gpu_delta import FP32_BAR, Case, check_backward, check_forward, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sla():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2401_00912_amd import sla as S

    S.lib()
    return S


ROWS = ("q", "k", "v", "g", "beta", "offsets")


def test_long_states_in_place(sla):
    """state_out in state_in, dstate_in in dstate_out, where a window is cut into parts: the first part's
    workgroup reads what the last one's writes."""
    import torch

    for dtype in ("f32", "bf16"):
        c = Case([2500, 70, 1400], 2, 4, 64, 64, dtype, seed=3, state=True, grads=True)
        args = [c.dev(x) for x in ROWS]
        o, st = c.forward(sla)
        g = sla.backward_delta(*args, c.dev("dout"), dstate=c.dev("dstate"), state=c.dev("state"))
        for _ in range(5):
            pool = c.dev("state")
            o2, _ = sla.forward_delta(*args, state=pool, final_state=pool)
            assert torch.equal(o, o2) and torch.equal(st, pool)
            ds, outs = c.dev("dstate"), [torch.empty_like(t) for t in args[:5]]
            need = sla.delta_backward_workspace_bytes(c.n, c.w, args[0].dtype, 2, 4, 64, 64)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            state, dout = c.dev("state"), c.dev("dout")
            code = {"f32": 0, "f16": 1, "bf16": 2}[dtype]
            p = lambda t: t.data_ptr()  # noqa: E731
            rc = sla.lib().sla_backward_delta(p(args[5]), c.n, c.w, None, code, 2, 4, 64, 64, c.scale, *map(p, args[:5]),
                                              p(state), p(dout), p(ds), *map(p, outs), p(ds), p(ws), need,
                                              torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            assert all(torch.equal(a, b) for a, b in zip(outs, g)) and torch.equal(ds, g[5])


@pytest.mark.parametrize("windows", [2, 40, 63, 64, 65])
def test_many_uneven_windows(sla, windows):
    """More workgroups than CUs (the longest windows first, up to 64 of them), with windows of the same length
    and without rows among them."""
    rng = np.random.default_rng(windows)
    lengths = rng.choice([0, 1, 17, 64, 65, 130, 200], size=windows).tolist()
    h = 8 if windows > 2 else 130
    check_forward(sla, Case(lengths, 2, h, 16, 16, "bf16", seed=windows, state=True, behind=3))
    check_backward(sla, Case(lengths, 2, h, 16, 16, "f32", seed=windows, state=True, behind=3, grads=True))


def test_many_windows_of_several_chunks(sla):
    """32 state rows and many workgroups: walks of several chunks that stage none ahead."""
    lengths = [200, 0, 129, 64, 65, 7] * 60
    check_forward(sla, Case(lengths, 3, 3, 32, 32, "f16", seed=1, state=True, order=True, behind=3))
    check_backward(sla, Case(lengths, 1, 3, 16, 80, "bf16", seed=2, state=True, order=True, behind=3, grads=True))


WRONG = ([0, 200, 100, 300, 250, 700], [-5, 300, 900, 10, 10, 2000], [700, 600, 500, 400, 0, 700],
         [0, 2000, 0, 2000, 0, 2000])


@pytest.mark.parametrize("fill", [0, 0x7f, 0xff])
@pytest.mark.parametrize("offsets", WRONG)
@pytest.mark.parametrize("n,dtype", [(700, "bf16"), (700, "f32"), (1500, "f16")])
def test_wrong_offsets_stay_in_range(sla, n, dtype, offsets, fill):
    """Offsets that are not in order, negative or past the end, rows' order past both ends, on a workspace
    full of something else: nothing before or behind the tensors is written, and the call ends."""
    import torch

    c = Case([n], 1, 2, 32, 48, dtype, seed=5, grads=True)
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    off = dev(offsets)
    order = torch.arange(n, dtype=torch.int32).cuda() * 3 - n
    args = [c.dev(x) for x in ROWS[:5]]
    w, dt = len(offsets) - 1, args[0].dtype
    for od in (None, order):
        guard = torch.full((3, n, 2, 48), 7.0, dtype=dt).cuda()
        ws = torch.full((sla.delta_workspace_bytes(n, w, dt, 1, 2, 32, 48),), fill, dtype=torch.uint8).cuda()
        sla.forward_delta(*args, off, order=od, out=guard[1], workspace=ws)
        ws = torch.full((sla.delta_backward_workspace_bytes(n, w, dt, 1, 2, 32, 48),), fill, dtype=torch.uint8).cuda()
        outs = [torch.full((3, *t.shape), 7.0, dtype=t.dtype).cuda() for t in args]
        sla.backward_delta(*args, off, c.dev("dout"), order=od, out=[t[1] for t in outs], workspace=ws)
        torch.cuda.synchronize()
        for t in (guard, *outs):
            assert (t[0] == 7.0).all() and (t[2] == 7.0).all()
    x = c.dev("v").reshape(n, 96)
    y = torch.full((3, n, 96), 7.0, dtype=dt).cuda()
    _, mean, rstd = sla.forward_group_norm(x, 4, offsets=off, y=y[1])
    dx = torch.full((3, n, 96), 7.0, dtype=dt).cuda()
    sla.backward_group_norm(x, 4, x, mean, rstd, offsets=off, dx=dx[1])
    torch.cuda.synchronize()
    for t in (y, dx):
        assert (t[0] == 7.0).all() and (t[2] == 7.0).all()


def test_workspace_contents_do_not_matter(sla):
    import torch

    for lengths, dtype in (([130, 1, 0, 64, 7], "bf16"), ([2600, 300], "f32"), ([2600, 300], "f16")):
        c = Case(lengths, 1, 2, 64, 48, dtype, seed=6, behind=5, order=True, grads=True)
        args, dt = [c.dev(x) for x in ROWS], c.dev("q").dtype
        got = []
        for fill in (0, 0xff, 0x7b):
            ws = torch.full((sla.delta_backward_workspace_bytes(c.n, c.w, dt, 1, 2, 64, 48),), fill,
                            dtype=torch.uint8).cuda()
            o = torch.zeros_like(args[2])
            outs = [torch.zeros_like(t) for t in args[:5]]
            _, st = c.forward(sla, out=o, workspace=ws)
            ws.fill_(fill)
            sla.backward_delta(*args, c.dev("dout"), order=c.dev("order"), out=outs, workspace=ws)
            got.append([o, st, *outs])
        for g in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got[0], g))


def layer(S, t, offsets, H, workspaces=None, outs=None):
    """A gated delta layer: o, the norm of its heads with an activation, and all gradients for dy."""
    import torch

    ws, out = workspaces or [None] * 4, outs or {}
    n = t["q"].shape[0]
    o, state = S.forward_delta(t["q"], t["k"], t["v"], t["g"], t["beta"], offsets, out=out.get("o"),
                               final_state=out.get("state"), workspace=ws[0])
    flat = o.view(n, -1)
    y, mean, rstd = S.forward_group_norm(flat, H, t["weight"], t["bias"], activation="silu", y=out.get("y"),
                                         mean=out.get("mean"), rstd=out.get("rstd"), workspace=ws[1])
    do, dw, db = S.backward_group_norm(flat, H, t["dy"], mean, rstd, t["weight"], t["bias"], activation="silu",
                                       dx=out.get("do"), workspace=ws[2])
    grads = S.backward_delta(t["q"], t["k"], t["v"], t["g"], t["beta"], offsets, do.view(o.shape), out=out.get("grads"),
                             workspace=ws[3])
    return [o, state, y, do, dw, db, *grads[:5]]


def layer_rows(dtype, lengths, hk=1, h=2, dk=32, dv=32, seed=0):
    import torch

    c = Case(lengths, hk, h, dk, dv, dtype, seed=seed, grads=True)
    gen = torch.Generator().manual_seed(seed + 100)
    t = {x: c.dev(x) for x in ROWS[:5]}
    t["dy"] = c.dev("dout").reshape(c.n, -1).contiguous()
    t["weight"] = (1 + 0.2 * torch.randn(h * dv, generator=gen)).cuda()
    t["bias"] = (0.2 * torch.randn(h * dv, generator=gen)).cuda()
    return c, t


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_layer_forward_and_backward(sla, dtype):
    """The operators one after the other, each against its reference on the inputs it was given."""
    c, t = layer_rows(dtype, [130, 1, 64, 77])
    o, state, y, do, dw, db, *grads = layer(sla, t, c.dev("offsets"), 2)
    wide = lambda x: x.double().cpu().numpy()  # noqa: E731
    ro, rs = c.forward_ref()
    close(o, ro, dtype, "o", FP32_BAR if dtype != "bf16" else 3 * 2.0 ** -11)
    close(state, rs, "f32", "state")
    flat = wide(o).reshape(c.n, -1)
    ry, rm, rr = delta_ref.group_norm_forward_ref(flat, 2, wide(t["weight"]), wide(t["bias"]), activation="silu")
    close(y, ry, dtype, "y")
    rdo, rdw, rdb = delta_ref.group_norm_backward_ref(flat, 2, wide(t["dy"]), rm, rr, wide(t["weight"]), wide(t["bias"]),
                                                      activation="silu")
    # a head's first rows can be small beside the rest: rstd is up to 1 / sqrt(eps) = 316 there, and so is what
    # a step of mean and rstd weighs; the limit is of the largest dx, which such a row makes
    close(do, rdo, dtype, "do")
    close(dw, rdw, "f32", "dweight")
    close(db, rdb, "f32", "dbias")
    ref = delta_ref.delta_backward_ref(*(c.wide(x) for x in ROWS[:5]), c.offsets, wide(do).reshape(c.n, 2, 32), c.scale)
    for name, got, want in zip(("dq", "dk", "dv", "dg", "dbeta"), grads, ref):
        own = name in ("dq", "dk") and dtype == "bf16"
        close(got, want, dtype if name in ("dq", "dk", "dv") else "f32", name, 1.5 * 2.0 ** -11 if own else FP32_BAR)


def test_layer_gradients_by_differences(sla):
    """The chain's gradients are those of the loss <y, dy>, in single precision."""
    import torch

    c, t = layer_rows("f32", [40, 90], seed=4)
    off = c.dev("offsets")

    def loss(t):
        o, _ = sla.forward_delta(t["q"], t["k"], t["v"], t["g"], t["beta"], off)
        y, _, _ = sla.forward_group_norm(o.view(c.n, -1), 2, t["weight"], t["bias"], eps=1e-2, activation="silu")
        return float((y.double() * t["dy"].double()).sum()), float(y.double().norm())

    o, _ = sla.forward_delta(t["q"], t["k"], t["v"], t["g"], t["beta"], off)
    flat = o.view(c.n, -1)
    _, mean, rstd = sla.forward_group_norm(flat, 2, t["weight"], t["bias"], eps=1e-2, activation="silu")
    do, dw, db = sla.backward_group_norm(flat, 2, t["dy"], mean, rstd, t["weight"], t["bias"], activation="silu")
    grads = sla.backward_delta(*(t[x] for x in ROWS[:5]), off, do.view(o.shape))
    gen = torch.Generator().manual_seed(9)
    for name, grad in zip((*ROWS[:5], "weight", "bias"), (*grads[:5], dw, db)):
        d = torch.randn(t[name].shape, generator=gen).cuda() * t[name].abs().mean()
        h = 1e-2
        (up, size), (down, _) = (loss({**t, name: t[name] + s * h * d}) for s in (1, -1))
        got, want = float((grad.double() * d.double()).sum()), (up - down) / (2 * h)
        # values are off by 1e-6 of their size, at random: of the loss by 1e-6 |y| |dy| / sqrt(values), and the
        # difference by its third derivative h^2
        noise = 1e-6 * size * float(t["dy"].double().norm()) / (c.n * 64) ** 0.5 / h
        scale = float((grad.double().norm() * d.double().norm()))
        assert abs(got - want) <= noise + 2e-3 * max(abs(want), 0.1 * scale), name


def test_scene_norm_behind_attention(sla):
    """Attention over a plan's windows, then the scenes' normalisation of its rows, and both backwards."""
    import torch


    gen = torch.Generator().manual_seed(1)
    n, W, H, d = 1200, 40, 4, 32
    win = torch.randint(0, W, (n,), generator=gen).to(torch.int32).cuda()
    plan = sla.build_segments(win, num_windows=W)
    q, k, v = (torch.randn(n, H, d, generator=gen).cuda() for _ in range(3))
    out = sla.forward(plan, q, k, v)
    scenes = torch.tensor([0, 500, 1150], dtype=torch.int32).cuda()
    x = out.reshape(n, H * d)
    y, mean, rstd = sla.forward_group_norm(x, 8, offsets=scenes, activation="relu", y=torch.zeros_like(x))
    ry, _, _ = delta_ref.group_norm_forward_ref(x.double().cpu().numpy(), 8, offsets=[0, 500, 1150], activation="relu")
    close(y, ry, "f32", "y")
    assert (y[1150:] == 0).all()
    # the same windows, row by row in their order
    r = [torch.nn.functional.normalize(t, dim=-1) for t in (q, k)]
    g, beta = -torch.rand(n, H, generator=gen).cuda(), torch.rand(n, H, generator=gen).cuda()
    _, perm, offs, _, _ = sla.read_plan(plan)
    o, _ = sla.forward_delta(*r, v, g, beta, plan.offsets, order=plan.perm)
    ro, _ = delta_ref.delta_forward_ref(*(t.double().cpu().numpy() for t in (*r, v, g, beta)), offs, d ** -0.5,
                                        order=perm)
    close(o, ro, "f32", "o")


@pytest.mark.parametrize("lengths,dtype", [([130, 1, 64, 77], "bf16"), ([2600, 300], "f32")])
def test_layer_in_a_graph(sla, lengths, dtype):
    """A captured layer (forward and backward) and single steps, replayed on new inputs with eager work
    between the replays: each replay is the eager result."""
    import torch

    c, t = layer_rows(dtype, lengths)
    off, dt, n = c.dev("offsets"), t["q"].dtype, c.n
    size = (n, c.w, dt, 1, 2, 32, 32)
    norm = lambda back: sla.group_norm_workspace_bytes(n, 0, dt, 64, 2, backward=back)  # noqa: E731
    ws = [torch.empty(b, dtype=torch.uint8, device="cuda")
          for b in (sla.delta_workspace_bytes(*size), norm(False), norm(True), sla.delta_backward_workspace_bytes(*size))]
    outs = dict(o=torch.zeros_like(t["v"]), state=torch.zeros(c.w, 2, 32, 32, device="cuda"), y=torch.zeros_like(t["dy"]),
                mean=torch.zeros(n, 2, device="cuda"), rstd=torch.zeros(n, 2, device="cuda"), do=torch.zeros_like(t["dy"]),
                grads=[torch.zeros_like(t[x]) for x in ROWS[:5]])
    pool = torch.zeros(4, 2, 32, 32, device="cuda")
    slots = torch.tensor([2, 0, 2, -1], dtype=torch.int32).cuda()
    step_out = torch.zeros_like(t["v"][:4])
    step = lambda: sla.step_delta(pool, slots, *(t[x][:4] for x in ROWS[:5]), out=step_out)  # noqa: E731
    layer(sla, t, off, 2, ws, outs)   # warm up
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer(sla, t, off, 2, ws, outs)
        step()
    for r in range(4):
        _, new = layer_rows(dtype, lengths, seed=10 + r)
        for x, y in new.items():
            t[x].copy_(y)
        pool.fill_(0.25 * r)
        step_out.zero_()
        want_state = pool.clone()
        want_step = sla.step_delta(want_state, slots, *(t[x][:4] for x in ROWS[:5]), out=torch.zeros_like(step_out))
        graph.replay()
        eager = layer(sla, t, off, 2)
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)
        assert torch.equal(pool, want_state) and torch.equal(step_out, want_step)


def test_two_streams(sla):
    """Two calls of everything at once, each on its own stream with its own workspaces, from inputs made there."""
    import torch

    lengths = [2600, 300, 64]
    want = []
    for i in range(2):
        c, t = layer_rows("bf16", lengths, seed=i)
        want.append((c, t, layer(sla, t, c.dev("offsets"), 2)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, (c, t, _) in zip(streams, want):
            with torch.cuda.stream(s):
                mine = {x: y.clone() for x, y in t.items()}
                got.append(layer(sla, mine, c.dev("offsets"), 2))
        torch.cuda.synchronize()
        for g, (_, _, w) in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_rows_past_two_billion_elements(sla):
    """q, k, v and their gradients of more than 2^31 elements each: the last windows are what they are alone."""
    import torch

    lengths = [1000] * 1050 + [300, 37]
    n, H, d = sum(lengths), 16, 128
    assert n * H * d > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(0)
    new = lambda: torch.randn(n, H, d, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    q, k, v, dout = new().mul_(d ** -0.5), new().mul_(d ** -0.5), new(), new()
    g, beta = -torch.rand(n, H, generator=gen, device="cuda"), torch.rand(n, H, generator=gen, device="cuda")
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
    last = torch.tensor([0, 300, 337], dtype=torch.int32).cuda()
    tail = [t[-337:].clone() for t in (q, k, v, g, beta)]
    o, st = sla.forward_delta(q, k, v, g, beta, off)
    o2, st2 = sla.forward_delta(*tail, last)
    assert torch.equal(o[-337:], o2) and torch.equal(st[-2:], st2)
    y, mean, rstd = sla.forward_group_norm(o.view(n, -1), H, activation="silu")
    y2, mean2, rstd2 = sla.forward_group_norm(o2.view(337, -1), H, activation="silu")
    assert torch.equal(y[-337:], y2) and torch.equal(mean[-337:], mean2)
    dx, _, _ = sla.backward_group_norm(o.view(n, -1), H, y, mean, rstd, activation="silu")
    dx2, _, _ = sla.backward_group_norm(o2.view(337, -1), H, y2, mean2, rstd2, activation="silu")
    assert torch.equal(dx[-337:], dx2)
    # one long window and a short one behind it: blocks of rows
    y, mean, _ = sla.forward_group_norm(o.view(n, -1), H, offsets=off[[0, 1050, 1051]].contiguous(), y=y)
    y2, mean2, _ = sla.forward_group_norm(o2[:300].view(300, -1), H, offsets=last[:2].contiguous())
    assert torch.allclose(mean[1], mean2[0], atol=1e-6) and torch.allclose(y[-337:-37].float(), y2.float(), rtol=2.0 ** -7,
                                                                         atol=1e-5)
    del y, y2, dx, o, o2
    grads = sla.backward_delta(q, k, v, g, beta, off, dout)
    grads2 = sla.backward_delta(*tail, last, dout[-337:].clone())
    for a, b in zip(grads[:5], grads2[:5]):
        assert torch.equal(a[-337:], b)


def test_states_past_two_billion_elements(sla):
    import torch

    slots, H, d = 8300, 16, 128
    assert slots * H * d * d > 2 ** 31
    pool = torch.empty(slots, H, d, d, device="cuda")
    gen = torch.Generator().manual_seed(2)
    use = [slots - 1, 0, 8200]
    small = torch.randn(3, H, d, d, generator=gen).cuda()
    for i, s in enumerate(use):
        pool[s] = small[i]
    c = Case([1] * 3, 16, 16, d, d, "bf16", seed=7)
    rows = [c.dev(x) for x in ROWS[:5]]
    o = sla.step_delta(pool, torch.tensor(use, dtype=torch.int32).cuda(), *rows)
    o2 = sla.step_delta(small, torch.arange(3, dtype=torch.int32).cuda(), *rows)
    assert torch.equal(o, o2) and all(torch.equal(pool[s], small[i]) for i, s in enumerate(use))


def test_order_may_name_a_row_twice(sla):
    """A row in two windows: each window is what it is with that row alone in it (o is one of the two)."""
    import torch

    c = Case([70, 70], 1, 1, 32, 32, "f32", seed=8)
    args = [c.dev(x) for x in ROWS]
    order = torch.cat([torch.arange(70), torch.arange(70)]).to(torch.int32).cuda()
    _, st = sla.forward_delta(*args, order=order)
    assert torch.equal(st[0], st[1])
