"""Performance cases of the gated delta rule and of group normalisation.

The gated delta rule is linear attention with a state that forgets and corrects itself.  For
every window (a sequence of consecutive rows) and value head, with a dk x dv state S that
starts at zero or at a given matrix, row by row in order:

    S   <- exp(g_t) S
    u_t  = beta_t (v_t - S^T k_t)
    S   <- S + k_t u_t^T
    o_t  = scale S^T q_t

Value head h reads query/key head h // (heads // heads_qk).  Group normalisation takes the mean
and variance of a window's rows over the channels of each group, then an affine map and an
activation; without windows every row is normalised by itself (one group per head: the norm
that follows the attention).

A case is a dict of
    kind       "delta_forward"   outputs and final states of all windows
               "delta_backward"  the gradients of everything the forward reads
               "delta_step"      one row for each of many sequences, states updated in place
               "norm_forward"    group normalisation and its statistics
               "norm_backward"   its gradients
    rows, dtype, spread          rows in all windows together, storage type, a seed-free shape number
    windows, layout              number of windows; "windows": rows of point-cloud windows (uneven,
                                 1 .. 144, some empty); "sequences": uneven long sequences;
                                 "rows": every row its own window (normalisation)
    heads_qk, heads, dk, dv      head counts and widths
    state                        an initial state is given (and, backward, the final state's gradient)
    channels, groups, activation of the normalisation
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CHUNK = 64
EPS = 1e-5


def _delta(name, kind, layout, rows, windows, heads_qk, heads, dk, dv, dtype, state=False, spread=0):
    c = dict(kind=kind, layout=layout, rows=rows, windows=windows, heads_qk=heads_qk, heads=heads, dk=dk, dv=dv,
             dtype=dtype, state=state, spread=spread)
    return c if name is None else dict(c, name=name)


def _norm(name, kind, layout, rows, windows, channels, groups, activation, dtype, spread=0):
    c = dict(kind=kind, layout=layout, rows=rows, windows=windows, channels=channels, groups=groups,
             activation=activation, dtype=dtype, spread=spread)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the windows of one LiDAR-like frame, 4 heads of 32: the rule in the place of the linear attention
        _delta("delta_windows_f16", "delta_forward", "windows", 59837, 1521, 4, 4, 32, 32, "f16"),
        # a batch of uneven sequences, two value heads to a key head
        _delta("delta_sequences_bf16", "delta_forward", "sequences", 12289, 7, 4, 8, 128, 128, "bf16"),
        # the largest forward: many sequences, wide heads
        _delta("delta_batch_bf16", "delta_forward", "sequences", 65536, 33, 16, 16, 128, 128, "bf16"),
        # one long sequence in single precision that goes on from a state
        _delta("delta_long_f32", "delta_forward", "sequences", 8191, 1, 4, 4, 64, 64, "f32", state=True),
        # a training step's gradients on the windows of a frame
        _delta("delta_windows_grad_f16", "delta_backward", "windows", 59837, 1521, 4, 4, 32, 32, "f16"),
        # and on uneven sequences with states in and out
        _delta("delta_sequences_grad_bf16", "delta_backward", "sequences", 16381, 9, 4, 8, 128, 128, "bf16", state=True),
        # answering one request, row by row: the smallest call
        _delta("delta_step_one_bf16", "delta_step", "rows", 1, 1, 2, 4, 64, 64, "bf16", state=True),
        # many requests at once
        _delta("delta_step_many_bf16", "delta_step", "rows", 256, 320, 8, 16, 128, 128, "bf16", state=True),
        # normalisation after a block on a batch of four frames
        _norm("norm_frames_bf16", "norm_forward", "sequences", 240011, 4, 256, 32, "silu", "bf16"),
        # the norm of the attention's output, head by head
        _norm("norm_heads_bf16", "norm_forward", "rows", 32768, 32768, 2048, 16, "none", "bf16"),
        # the gradients on one frame
        _norm("norm_frame_grad_f16", "norm_backward", "sequences", 59837, 1, 128, 8, "relu", "f16"),
        # and on short windows, each with statistics of its own
        _norm("norm_windows_grad_f32", "norm_backward", "windows", 59837, 1521, 128, 4, "silu", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    spread = rng.randrange(1 << 20)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    kind = rng.choice(["delta_forward", "delta_forward", "delta_backward", "delta_backward", "delta_step",
                       "norm_forward", "norm_backward"])
    if kind.startswith("norm"):
        layout = rng.choice(["sequences", "windows", "rows"])
        width, groups = rng.choice([4, 8, 16, 24, 32, 64, 128]), rng.choice([1, 2, 4, 8, 16, 32])
        while not 32 <= width * groups <= 2048:
            width, groups = rng.choice([4, 8, 16, 24, 32, 64, 128]), rng.choice([1, 2, 4, 8, 16, 32])
        channels = width * groups
        rows = _log_int(rng, 1, 60000000 // channels // (2 if kind == "norm_backward" else 1))
        rows = min(rows, 240000)
        windows = {"sequences": min(rows, rng.randint(1, 6)), "windows": max(1, rows // 40), "rows": rows}[layout]
        return _norm(None, kind, layout, rows, windows, channels, groups, rng.choice(["none", "relu", "silu"]), dtype,
                     spread)
    heads_qk, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4])
    dk, dv = rng.choice([16, 32, 48, 64, 128, 128]), rng.choice([16, 32, 64, 96, 128, 128])
    heads = heads_qk * group
    if kind == "delta_step":
        rows = _log_int(rng, 1, min(256, 256 * 16 * 128 * 128 // (heads * dk * dv)))
        return _delta(None, kind, "rows", rows, rows + rng.randint(0, 20), heads_qk, heads, dk, dv, dtype, True, spread)
    layout = rng.choice(["sequences", "sequences", "windows"])
    most = 24576 * 2048 // (heads * max(dk, dv)) // (4 if kind == "delta_backward" else 1) // (2 if dtype == "f32" else 1)
    rows = _log_int(rng, 1, min(most, 65536 if layout == "windows" else 32768))
    windows = max(1, rows // 40) if layout == "windows" else min(rows, _log_int(rng, 1, 40))
    return _delta(None, kind, layout, rows, windows, heads_qk, heads, dk, dv, dtype, rng.random() < 0.5, spread)


def _lengths(case, seed):
    """Rows of every window, uneven, some zero: a list whose sum is the case's rows."""
    n, w = case["rows"], case["windows"]
    if case["layout"] == "rows":
        return [1] * n
    rng = random.Random(1000003 * seed + case["spread"])
    sigma = 0.7 if case["layout"] == "windows" else 1.0
    share = [0.0 if w > 2 and rng.random() < 0.05 else rng.lognormvariate(0.0, sigma) for _ in range(w)]
    share[rng.randrange(w)] += 1e-9
    most = 144 if case["layout"] == "windows" and n <= 100 * w else n
    total = sum(share)
    lengths = [min(most, int(n * s / total)) for s in share]
    left = n - sum(lengths)
    while left > 0:
        i = rng.randrange(w)
        more = min(left, most - lengths[i], max(1, left // 8))
        lengths[i] += more
        left -= more
    return lengths


def prepare(case, seed):
    dev, dt = "cuda", DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
    n = case["rows"]
    s = dict(case=case)
    if case["kind"] != "delta_step":
        s["lengths"] = _lengths(case, seed)
        s["offsets"] = torch.tensor([0] + s["lengths"], dtype=torch.int64).cumsum(0).to(torch.int32).to(dev)
    if case["kind"].startswith("norm"):
        C = case["channels"]
        s["x"] = (normal(n, C) * (0.5 + torch.rand(C, device=dev, generator=gen)) + 0.5 * normal(C)).to(dt)
        s["weight"], s["bias"] = 1 + 0.2 * normal(C), 0.2 * normal(C)
        if case["kind"] == "norm_backward":
            s["dy"] = normal(n, C).to(dt)
            # the forward's statistics, which a training step has kept
            s["mean"], s["rstd"] = _plain_stats(s)
        return s
    hk, hv, dk, dv = case["heads_qk"], case["heads"], case["dk"], case["dv"]
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    silu = torch.nn.functional.silu
    # rows as the layers make them: queries and keys pass an activation and are normalised, a
    # log decay per head that spans slow to fast forgetting, a sigmoid as the writing strength
    s["q"], s["k"] = unit(silu(normal(n, hk, dk))).to(dt), unit(silu(normal(n, hk, dk))).to(dt)
    s["v"] = normal(n, hv, dv).to(dt)
    rate = torch.exp(torch.empty(hv, device=dev).uniform_(-4.0, 1.0, generator=gen))
    s["g"] = -rate * torch.nn.functional.softplus(normal(n, hv))
    s["beta"] = torch.sigmoid(normal(n, hv))
    s["scale"] = dk ** -0.5
    if case["kind"] == "delta_step":
        s["state"] = 0.3 * normal(case["windows"], hv, dk, dv)
        slots = torch.randperm(case["windows"], device=dev, generator=gen)[:n].to(torch.int32)
        s["slots"] = slots
        return s
    w = case["windows"]
    s["state"] = 0.3 * normal(w, hv, dk, dv) if case["state"] else None
    if case["kind"] == "delta_backward":
        s["dout"] = normal(n, hv, dv).to(dt)
        s["dstate"] = 0.3 * normal(w, hv, dk, dv) if case["state"] else None
    return s


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2401_00912_amd import sla

    case, kind = s["case"], s["case"]["kind"]
    if kind == "delta_forward":
        return sla.forward_delta(s["q"], s["k"], s["v"], s["g"], s["beta"], s["offsets"], scale=s["scale"],
                                 state=s["state"])
    if kind == "delta_backward":
        return [t for t in sla.backward_delta(s["q"], s["k"], s["v"], s["g"], s["beta"], s["offsets"], s["dout"],
                                              scale=s["scale"], state=s["state"], dstate=s["dstate"])
                if t is not None]
    if kind == "delta_step":
        return sla.step_delta(s["state"], s["slots"], s["q"], s["k"], s["v"], s["g"], s["beta"],
                              scale=s["scale"]), s["state"]
    offsets = None if case["layout"] == "rows" else s["offsets"]
    if kind == "norm_forward":
        return sla.forward_group_norm(s["x"], case["groups"], weight=s["weight"], bias=s["bias"], offsets=offsets,
                                      eps=EPS, activation=case["activation"])
    return sla.backward_group_norm(s["x"], case["groups"], s["dy"], s["mean"].contiguous(), s["rstd"].contiguous(),
                                   weight=s["weight"], bias=s["bias"], offsets=offsets, activation=case["activation"])


# ------------------------------------------------------------------ the plain forms
def _chunks(s):
    """Chunks of at most 64 rows: their rows [chunks, 64], which of these exist, for every window its
    first chunk and chunk count, windows with more chunks first."""
    dev = s["q"].device
    lens = torch.tensor(s["lengths"], dtype=torch.int64)
    counts = (lens + CHUNK - 1) // CHUNK
    by = torch.argsort(counts, descending=True, stable=True)
    starts = torch.cumsum(lens, 0) - lens
    first = torch.cumsum(counts, 0) - counts
    win = torch.repeat_interleave(torch.arange(lens.numel()), counts)
    at = torch.arange(win.numel()) - first[win]
    rows = (starts[win] + at * CHUNK)[:, None] + torch.arange(CHUNK)[None, :]
    real = rows < (starts + lens)[win][:, None]
    rows = torch.where(real, rows, torch.zeros_like(rows))
    return rows.to(dev), real.to(dev), by.to(dev), first[by].to(dev), counts[by].tolist()


def _gathered(s, names, rows, real):
    """float32 [chunks, heads, 64, width] of the rows, zero where there is none; keys and queries once
    for every value head."""
    hv = s["v"].shape[1]
    got = []
    for name in names:
        x = s[name].float()
        x = x[:, :, None] if x.dim() == 2 else x
        x = x.repeat_interleave(hv // x.shape[1], dim=1)
        got.append((x[rows] * real[:, :, None, None]).transpose(1, 2).contiguous())
    return got


def _decays(g):
    """exp of the summed log decays between two rows of a chunk, from its start and to its end."""
    gam = g[..., 0].double().cumsum(-1)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=g.device).tril()
    between = torch.exp((gam[..., :, None] - gam[..., None, :]).masked_fill(~lower, -math.inf))
    return between.float(), torch.exp(gam).float(), torch.exp(gam[..., -1:] - gam).float()


def _inverse(a):
    """(I + a)^-1 for strictly lower triangular a, row by row."""
    t = torch.zeros_like(a)
    t += torch.eye(CHUNK, device=a.device)
    for i in range(1, CHUNK):
        t[..., i, :i] = -(a[..., i:i + 1, :i] @ t[..., :i, :i].contiguous())[..., 0, :]
    return t


def _plain_scan(s, want_states=False):
    rows, real, by, first, counts = _chunks(s)
    q, k, v, g, b = _gathered(s, ("q", "k", "v", "g", "beta"), rows, real)
    between, since, until = _decays(g)
    kt = k.transpose(-1, -2).contiguous()
    kk = k @ kt
    strict = torch.ones(CHUNK, CHUNK, device=k.device).tril(-1)
    t = _inverse(b * between * kk * strict)
    w = t @ (b * since[..., None] * k)
    u0 = t @ (b * v)
    p = s["scale"] * between * (q @ kt)
    n_windows, hv, dk, dv = len(s["lengths"]), v.shape[1], k.shape[-1], v.shape[-1]
    state = torch.zeros(n_windows, hv, dk, dv, device=k.device)
    if s["state"] is not None:
        state += s["state"].float()[by]
    states = torch.empty(rows.shape[0], hv, dk, dv, device=k.device)
    u = torch.empty_like(u0)
    for c in range(counts[0] if counts else 0):
        m = sum(x > c for x in counts)
        at = first[:m] + c
        states[at] = state[:m]
        u[at] = u0[at] - w[at] @ state[:m]
        state[:m] = since[at][..., -1, None, None] * state[:m] + (kt[at] * until[at][..., None, :]) @ u[at]
    out = torch.empty_like(state)
    out[by] = state
    o = s["scale"] * since[..., None] * (q @ states) + p @ u
    if not want_states:
        return rows, real, o, out
    return rows, real, by, first, counts, q, k, v, b, g, between, since, until, kk, t, w, p, u, states, o, out


def _put(rows, real, x, like):
    y = torch.zeros(like.shape[0], *x.shape[1:2], *x.shape[3:], device=x.device, dtype=x.dtype)
    y[rows[real]] = x.transpose(1, 2)[real]
    return y


def _plain_delta_forward(s):
    rows, real, o, state = _plain_scan(s)
    return _put(rows, real, o, s["v"]).to(s["v"].dtype), state


def _plain_delta_backward(s):
    (rows, real, by, first, counts, q, k, v, b, g, between, since, until, kk, t, w, p, u, states, o,
     _) = _plain_scan(s, True)
    scale = s["scale"]
    do, = _gathered(s, ("dout",), rows, real)
    tr = lambda x: x.transpose(-1, -2).contiguous()  # noqa: E731
    strict = torch.ones(CHUNK, CHUNK, device=k.device).tril(-1)
    du0 = tr(p) @ do
    qd = tr(scale * since[..., None] * q) @ do
    wt = tr(w)
    kd = until[..., None] * k
    ds = torch.zeros(len(s["lengths"]), *states.shape[1:], device=k.device)
    if s["dstate"] is not None:
        ds += s["dstate"].float()[by]
    dstates = torch.empty_like(states)
    du = torch.empty_like(u)
    for c in range((counts[0] if counts else 0) - 1, -1, -1):
        m = sum(x > c for x in counts)
        at = first[:m] + c
        dstates[at] = ds[:m]
        du[at] = du0[at] + kd[at] @ ds[:m]
        ds[:m] = qd[at] + since[at][..., -1, None, None] * ds[:m] - wt[at] @ du[at]
    dstate_in = torch.empty_like(ds)
    dstate_in[by] = ds
    dx = tr(t) @ du
    st = tr(states)
    dp = (do @ tr(u)) * between * scale
    dm = -(dx @ tr(u)) * between * strict  # with respect to beta_i k_i . k_j
    bk = (b * dm)
    dq_state = scale * since[..., None] * (do @ st)
    dq = dq_state + dp @ k
    dk_row = bk @ k - b * since[..., None] * (dx @ st)
    dk_in = until[..., None] * (u @ tr(dstates))
    dk_col = tr(bk) @ k + tr(dp) @ q + dk_in
    dv = b * dx
    resid = v - since[..., None] * (k @ states)
    db = (dx * resid).sum(-1) + (dm * kk).sum(-1)
    dgam = (q * dq).sum(-1) + (k * dk_row).sum(-1) - (k * dk_col).sum(-1)
    last = (k * dk_in).sum((-1, -2)) + since[..., -1] * (states * dstates).sum((-1, -2))
    dgam[..., -1] += last
    dg = dgam.double().flip(-1).cumsum(-1).flip(-1).float()
    hk, hv = s["q"].shape[1], s["v"].shape[1]
    dt = s["v"].dtype
    shared = lambda x: x.view(x.shape[0], hk, hv // hk, x.shape[-1]).sum(2)  # noqa: E731
    got = [shared(_put(rows, real, dq, s["v"])).to(dt), shared(_put(rows, real, dk_row + dk_col, s["v"])).to(dt),
           _put(rows, real, dv, s["v"]).to(dt), _put(rows, real, dg[..., None], s["v"])[..., 0],
           _put(rows, real, db[..., None], s["v"])[..., 0]]
    if s["state"] is not None:
        got.append(dstate_in)
    return got


def _plain_step(s):
    hv = s["v"].shape[1]
    wide = lambda x: x.float().repeat_interleave(hv // x.shape[1], dim=1)  # noqa: E731
    at = s["slots"].long()
    q, k, v = wide(s["q"]), wide(s["k"]), s["v"].float()
    state = torch.exp(s["g"])[..., None, None] * s["state"][at]
    u = s["beta"][..., None] * (v - (state * k[..., None]).sum(-2))
    state = state + k[..., None] * u[..., None, :]
    s["state"][at] = state
    return (s["scale"] * (state * q[..., None]).sum(-2)).to(s["v"].dtype), s["state"]


def _segments(s):
    w = torch.tensor(s["lengths"], dtype=torch.int64, device=s["x"].device)
    return torch.repeat_interleave(torch.arange(w.numel(), device=w.device), w, output_size=s["x"].shape[0]), w


def _sums(s, x):
    """Sums of the consecutive rows of every window, as differences of running sums in 64 bits."""
    run = torch.nn.functional.pad(x.t().contiguous().cumsum(-1), (1, 0))
    at = s["offsets"].long()
    return (run[:, at[1:]] - run[:, at[:-1]]).t()


def _plain_stats(s):
    """Mean and 1 / sqrt(variance + eps) of every window and group, from sums in 64 bits."""
    x, G = s["x"], s["case"]["groups"]
    x = x.view(x.shape[0], G, -1).double()
    if s["case"]["layout"] == "rows":
        mean = x.mean(-1)
        var = (x - mean[..., None]).square().mean(-1)
    else:
        seg, count = _segments(s)
        count = (count * x.shape[-1]).clamp(min=1)[:, None].double()
        mean = _sums(s, x.sum(-1)) / count
        var = _sums(s, (x - mean[seg][..., None]).square().sum(-1)) / count
    return mean.float(), torch.rsqrt(var + EPS).float()


def _spread(s, stat):
    return stat if s["case"]["layout"] == "rows" else stat[_segments(s)[0]]


def _activation(name, z):
    return z if name == "none" else z.clamp(min=0) if name == "relu" else z * torch.sigmoid(z)


def _slope(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).float()
    sig = torch.sigmoid(z)
    return sig * (1 + z * (1 - sig))


def _plain_norm_forward(s):
    x, G = s["x"], s["case"]["groups"]
    n, C = x.shape
    mean, rstd = _plain_stats(s)
    hat = ((x.float().view(n, G, -1) - _spread(s, mean)[..., None]) * _spread(s, rstd)[..., None]).view(n, C)
    return _activation(s["case"]["activation"], hat * s["weight"] + s["bias"]).to(x.dtype), mean, rstd


def _plain_norm_backward(s):
    x, G = s["x"], s["case"]["groups"]
    n, C = x.shape
    rstd = _spread(s, s["rstd"])
    hat = (x.float().view(n, G, -1) - _spread(s, s["mean"])[..., None]) * rstd[..., None]
    dz = s["dy"].float() * _slope(s["case"]["activation"], hat.view(n, C) * s["weight"] + s["bias"])
    dw = (dz * hat.view(n, C)).double().sum(0).float()
    db = dz.double().sum(0).float()
    dhat = (dz * s["weight"]).view(n, G, -1)
    a, b = dhat.double().sum(-1), (dhat * hat).double().sum(-1)
    if s["case"]["layout"] == "rows":
        a, b = a / (C // G), b / (C // G)
    else:
        seg, count = _segments(s)
        count = (count * (C // G)).clamp(min=1)[:, None].double()
        a, b = (_sums(s, a) / count)[seg], (_sums(s, b) / count)[seg]
    dx = rstd[..., None] * (dhat - a.float()[..., None] - hat * b.float()[..., None])
    return dx.view(n, C).to(x.dtype), dw, db


def run(s):
    if own:
        return _own(s)
    return {"delta_forward": _plain_delta_forward, "delta_backward": _plain_delta_backward, "delta_step": _plain_step,
            "norm_forward": _plain_norm_forward, "norm_backward": _plain_norm_backward}[s["case"]["kind"]](s)


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_delta_forward(s, keep=None):
    """Row by row, all windows side by side, the longest first.  keep: collects the states before every
    64th row."""
    q, k, v, g, b = (s[x].double() for x in ("q", "k", "v", "g", "beta"))
    hv = v.shape[1]
    q, k = (x.repeat_interleave(hv // x.shape[1], dim=1) for x in (q, k))
    order = sorted(range(len(s["lengths"])), key=lambda i: -s["lengths"][i])
    lens = [s["lengths"][i] for i in order]
    start = s["offsets"].long()[:-1][torch.tensor(order, device=q.device)]
    S = torch.zeros(len(order), hv, k.shape[-1], v.shape[-1], dtype=torch.float64, device=q.device)
    if s["state"] is not None:
        S = s["state"].double()[torch.tensor(order, device=q.device)]
    o = torch.zeros_like(v)
    m = len(order)
    for t in range(lens[0]):
        while lens[m - 1] <= t:
            m -= 1
        if keep is not None and t % 64 == 0:
            keep.append(S[:m].clone())
        r = start[:m] + t
        A = S[:m] * torch.exp(g[r])[..., None, None]
        u = b[r][..., None] * (v[r] - torch.matmul(k[r][..., None, :], A)[..., 0, :])
        A += k[r][..., :, None] * u[..., None, :]
        S[:m] = A
        o[r] = s["scale"] * torch.matmul(q[r][..., None, :], A)[..., 0, :]
    out = torch.empty_like(S)
    out[torch.tensor(order, device=q.device)] = S
    return o, out


def _exact_delta_backward(s):
    """The chain rule of one row, from the last row to the first, on states made again from every 64th."""
    keep = []
    _exact_delta_forward(s, keep)
    q, k, v, g, b, do = (s[x].double() for x in ("q", "k", "v", "g", "beta", "dout"))
    hk, hv = q.shape[1], v.shape[1]
    q, k = (x.repeat_interleave(hv // hk, dim=1) for x in (q, k))
    order = sorted(range(len(s["lengths"])), key=lambda i: -s["lengths"][i])
    lens = [s["lengths"][i] for i in order]
    at = torch.tensor(order, device=q.device)
    start = s["offsets"].long()[:-1][at]
    dS = torch.zeros(len(order), hv, k.shape[-1], v.shape[-1], dtype=torch.float64, device=q.device)
    if s["dstate"] is not None:
        dS = s["dstate"].double()[at]
    dq, dk, dv, dg, db = (torch.zeros_like(x) for x in (q, k, v, g, b))
    alive = lambda t: sum(x > t for x in lens)  # noqa: E731
    for c in range(len(keep) - 1, -1, -1):
        hi = min(lens[0], 64 * c + 64)
        S, before = keep[c].clone(), []
        for t in range(64 * c, hi):
            m = alive(t)
            r = start[:m] + t
            before.append(S[:m].clone())
            A = S[:m] * torch.exp(g[r])[..., None, None]
            u = b[r][..., None] * (v[r] - torch.matmul(k[r][..., None, :], A)[..., 0, :])
            S = A + k[r][..., :, None] * u[..., None, :]
        for t in range(hi - 1, 64 * c - 1, -1):
            P = before.pop()
            m = P.shape[0]
            r = start[:m] + t
            al = torch.exp(g[r])[..., None, None]
            A = P * al
            e = v[r] - torch.matmul(k[r][..., None, :], A)[..., 0, :]
            u = b[r][..., None] * e
            N = A + k[r][..., :, None] * u[..., None, :]
            dq[r] = s["scale"] * torch.matmul(N, do[r][..., None])[..., 0]
            D = dS[:m] + s["scale"] * q[r][..., :, None] * do[r][..., None, :]
            du = torch.matmul(k[r][..., None, :], D)[..., 0, :]
            de = b[r][..., None] * du
            db[r] = (du * e).sum(-1)
            dv[r] = de
            dk[r] = torch.matmul(D, u[..., None])[..., 0] - torch.matmul(A, de[..., None])[..., 0]
            D = D - k[r][..., :, None] * de[..., None, :]
            dg[r] = (D * A).sum((-1, -2))
            dS[:m] = D * al
    d0 = torch.empty_like(dS)
    d0[at] = dS
    shared = lambda x: x.view(x.shape[0], hk, hv // hk, x.shape[-1]).sum(2)  # noqa: E731
    got = [shared(dq), shared(dk), dv, dg, db]
    return got + [d0] if s["state"] is not None else got


def _exact_step(s):
    o = torch.empty(s["v"].shape, dtype=torch.float64, device=s["v"].device)
    state = s["state"].double()
    group = s["v"].shape[1] // s["q"].shape[1]
    at = s["slots"].long()
    for h in range(s["v"].shape[1]):
        q, k, v = s["q"][:, h // group].double(), s["k"][:, h // group].double(), s["v"][:, h].double()
        A = state[at, h] * torch.exp(s["g"][:, h].double())[:, None, None]
        u = s["beta"][:, h, None].double() * (v - (A.transpose(1, 2) @ k[..., None])[..., 0])
        A = A + k[:, :, None] * u[:, None, :]
        state[at, h] = A
        o[:, h] = s["scale"] * (A.transpose(1, 2) @ q[..., None])[..., 0]
    return o, state


def _exact_norm(s):
    case = s["case"]
    C, G = case["channels"], case["groups"]
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    grad = case["kind"] == "norm_backward"
    if grad:
        dy, mean, rstd = s["dy"].double(), s["mean"].double(), s["rstd"].double()
        dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(b)
    else:
        y, means, rstds = torch.zeros_like(x), [], []
    # every row by itself: one block in which a row is a window; else window by window
    blocks = [(0, x.shape[0], True)] if case["layout"] == "rows" else []
    if not blocks:
        begin = 0
        for i, m in enumerate(s["lengths"]):
            blocks.append((begin, begin + m, False))
            begin += m
    for i, (lo, hi, single) in enumerate(blocks):
        X = x[lo:hi].view(hi - lo, G, C // G)
        dims = (2,) if single else (0, 2)
        if grad:
            M, R = (mean, rstd) if single else (mean[i][None], rstd[i][None])
        elif hi == lo:
            M, R = torch.zeros(1, G, dtype=x.dtype, device=x.device), torch.full((1, G), EPS, dtype=x.dtype,
                                                                                   device=x.device).rsqrt()
        else:
            M = X.mean(dims).view(-1, G)
            R = (X - M[..., None]).square().mean(dims).view(-1, G).add(EPS).rsqrt()
        hat = (X - M[..., None]) * R[..., None]
        z = hat.reshape(hi - lo, C) * w + b
        gate = torch.sigmoid(z) if case["activation"] == "silu" else (z > 0).double() if case["activation"] == "relu" \
            else torch.ones_like(z)
        if not grad:
            y[lo:hi] = z * gate
            means.append(M)
            rstds.append(R)
            continue
        dz = dy[lo:hi] * (gate + z * gate * (1 - gate) if case["activation"] == "silu" else gate)
        H = hat.reshape(hi - lo, C)
        dw += (dz * H).sum(0)
        db += dz.sum(0)
        dh = (dz * w).view(hi - lo, G, C // G)
        if hi > lo:
            dx[lo:hi] = (R[..., None] * (dh - dh.mean(dims, keepdim=True) - hat * (dh * hat).mean(dims, keepdim=True))
                         ).reshape(hi - lo, C)
    return (dx, dw, db) if grad else (y, torch.cat(means), torch.cat(rstds))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "delta_forward":
        return _exact_delta_forward(s)
    if kind == "delta_backward":
        return _exact_delta_backward(s)
    if kind == "delta_step":
        return _exact_step(s)
    return _exact_norm(s)


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    n, w = case["rows"], case["windows"]
    if case["kind"].startswith("norm"):
        values, stats = n * case["channels"], 8 * w * case["groups"]
        if case["kind"] == "norm_forward":
            return {"bytes": 2 * values * size + stats + 8 * case["channels"], "flops": 8 * values}
        return {"bytes": 3 * values * size + stats + 16 * case["channels"], "flops": 16 * values}
    hk, hv, dk, dv = case["heads_qk"], case["heads"], case["dk"], case["dv"]
    rows = n * (2 * hk * dk + 2 * hv * dv) * size + 8 * n * hv
    state = 4 * hv * dk * dv
    # three products of a state with a vector for each row and head; the gradients: six, and two to
    # make the states again
    if case["kind"] == "delta_forward":
        return {"bytes": rows + (2 if case["state"] else 1) * w * state, "flops": 6 * n * hv * dk * dv}
    if case["kind"] == "delta_step":
        return {"bytes": rows + 2 * n * state + 4 * n, "flops": 7 * n * hv * dk * dv}
    return {"bytes": n * (4 * hk * dk + 3 * hv * dv) * size + 16 * n * hv + (3 * w * state if case["state"] else 0),
            "flops": 16 * n * hv * dk * dv}
