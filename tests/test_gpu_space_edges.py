"""The short convolution's and the selective scan's edges: orders that name no row, workspaces of just the bytes that
are needed, and the sizes at which a call goes another way (two channels a lane in single rows, long parts, many
windows), against the float64 reference.
Tolerances are those of the operators' own tests.  A parameter's gradient is summed by a lane over a part's rows, over
a sixteenth of the parts and over sixteen of those sums, so by at most rows + parts / 16 + 16 roundings of 2^-24 of the
terms' sizes: with parts of 64 rows and up to 520 parts 6.7e-6, which leaves the terms' own 2e-6 below 1e-5; with
parts of 128 rows and up to 170 of them 9.3e-6, so that 1.5e-5 is the limit there."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import space_ref
from tests.gpu_util import torch_dtype
from tests.test_gpu_conv import Case as ConvCase
from tests.test_gpu_conv import close, within
from tests.test_gpu_scan import OPTIONS, Case

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


# ------------------------------------------------------------------ short convolution
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("C", [9, 24, 64])
def test_an_order_that_names_no_row_is_a_row_of_zeros(sla, dtype, C, K):
    """Forward and gradients of the same function: a position whose order is out of range is a row of zeros whose
    result is not written and has no gradient."""
    import torch

    c = ConvCase([40, 3, 0, 17], C, K, dtype, seed=31, state=True, order=True)
    bad = [0, 5, 6, 20, 39, 41, 43, 59]
    c.order[bad] = torch.tensor([-1, c.n, 2 ** 31 - 1, -2 ** 31] * 2, dtype=torch.int32, device="cuda")
    h = c.host
    zero = lambda t: np.concatenate([t, np.zeros((1, C))])  # noqa: E731
    order = c.ref_kw["order"].copy()
    order[bad] = c.n
    kw = {**c.ref_kw, "order": order}
    y, st = sla.forward_short_conv(c.x, c.weight, c.off, y=c.new(), **c.kw)
    ry, rs = space_ref.conv_forward_ref(zero(h["x"]), h["w"], c.offsets, **kw)
    close(y, ry[:-1], dtype, "y")
    assert (num(st) == rs).all()
    dx, dw, db, ds = sla.backward_short_conv(c.x, c.weight, c.off, c.dy, dstate=c.dstate, dx=c.new(), **c.kw)
    gx, gw, gb, gs = space_ref.conv_backward_ref(zero(h["x"]), h["w"], c.offsets, zero(h["dy"]), dstate=h["d"], **kw)
    close(dx, gx[:-1], dtype, "dx")
    close(ds, gs, dtype, "dstate_in")
    _, sw, sb, _ = space_ref.conv_backward_ref(np.abs(zero(h["x"])), np.zeros_like(h["w"]), c.offsets, np.abs(zero(h["dy"])),
                                               activation="none", state=np.abs(h["s"]), order=order)
    within(dw, gw, 1.1 * 2.0e-5 * sw, "dweight")
    within(db, gb, 1.1 * 2.0e-5 * sb, "dbias")


# ------------------------------------------------------------------ workspaces
@pytest.mark.parametrize("n,W", [(159, 1), (160, 3), (160, 4), (255, 2), (256, 8), (383, 1), (384, 1), (575, 1), (576, 3),
                                 (640, 5), (1024, 2), (1100, 4)])
def test_calls_stay_in_their_workspace(sla, n, W):
    """Workspaces of just the bytes asked for, at the widths whose cuts change with these rows and windows, and one of
    more rows and windows for the same calls: the bytes beside them stay, the results are the same."""
    import torch

    D = 65536
    gen = torch.Generator(device="cuda").manual_seed(n)
    rows = lambda *s: torch.randn(*s, device="cuda", generator=gen).half()  # noqa: E731
    x, delta, dy, B, C = rows(n, D), rows(n, D), rows(n, D), rows(n, 1, 1), rows(n, 1, 1)
    A, weight = -torch.ones(D, 1, device="cuda"), torch.randn(D, 2, device="cuda", generator=gen)
    cuts = sorted(torch.randint(0, n + 1, (W - 1,), generator=torch.Generator().manual_seed(n)).tolist())
    off = torch.tensor([0, *cuts, n], dtype=torch.int32, device="cuda")

    def run(need, f):
        buf = torch.full((need + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
        got = f(buf[4096:-4096])
        torch.cuda.synchronize()
        assert (buf[:4096] == 0x5A).all() and (buf[-4096:] == 0x5A).all()
        return [t for t in got if t is not None]

    for need, f in (
            (lambda n, W: sla.short_conv_backward_workspace_bytes(n, W, x.dtype, D, 2),
             lambda ws: sla.backward_short_conv(x, weight, off, dy, workspace=ws)),
            (lambda n, W: sla.selective_scan_workspace_bytes(n, W, x.dtype, D, 1, 1),
             lambda ws: sla.forward_selective_scan(x, delta, A, B, C, off, delta_softplus=True, workspace=ws)),
            (lambda n, W: sla.selective_scan_backward_workspace_bytes(n, W, x.dtype, D, 1, 1),
             lambda ws: sla.backward_selective_scan(x, delta, A, B, C, off, dy, delta_softplus=True, workspace=ws))):
        a, b = run(need(n, W), f), run(need(n + 37, W + 5), f)
        assert all(torch.equal(p, q) for p, q in zip(a, b))


# ------------------------------------------------------------------ selective scan
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [1, 3, 8, 16, 32, 64])
def test_an_order_that_names_no_row_is_left_out(sla, dtype, N, gate):
    """As if the windows were without these positions: states go past them, and no other row knows."""
    import torch

    c = Case([70, 3, 0, 150], 72, N, dtype, 2, seed=32, state=True, order=True, gate=gate)
    bad = [0, 5, 6, 7, 8, 69, 71, 73, 222, 100, 101, 102]   # in all four places of a batch, at parts' ends too
    order = c.ref_kw["order"]
    c.order[bad] = torch.tensor([-1, c.n, 2 ** 31 - 1, -2 ** 31] * 3, dtype=torch.int32, device="cuda")
    kept = [[p for p in range(lo, hi) if p not in bad] for lo, hi in zip(c.offsets[:-1], c.offsets[1:])]
    c.ref_kw["order"] = order[sum(kept, [])]
    c.offsets = np.cumsum([0] + [len(k) for k in kept])
    c.forward(sla)
    c.backward(sla)


# 256 rows and more: two channels a lane from n channels LN = 2^20 on, LN the lanes of a channel
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,D,N", [(256, 1030, 16), (255, 1028, 16), (256, 4096, 5), (100, 1031, 64), (257, 4100, 4),
                                   (70, 3001, 24)])
def test_many_single_rows(sla, dtype, n, D, N):
    import torch

    gen = torch.Generator().manual_seed(n + D)
    slots = torch.randint(0, n, (n,), generator=gen).to(torch.int32)   # some twice and more
    slots[::17], slots[5::31] = -1, n + 3                              # and some that are none
    for strided in (False, True):
        c = Case([n], D, N, dtype, seed=D, strided=strided)
        pool = torch.randn(n, D, N, generator=gen).cuda()
        opts = {k: c.r[k] for k in OPTIONS}
        ry, rs = space_ref.scan_step_ref(num(pool), slots.numpy(), *map(num, c.args()), **{k: num(v) for k, v in opts.items()},
                                         delta_softplus=True)
        y = sla.step_selective_scan(pool, slots.cuda(), *c.args(), **opts, delta_softplus=True, y=c.new(c.r["x"]))
        close(y, ry, dtype, "y")
        close(pool, rs, "f32", "state")


def uneven(W, mean, longest, seed):
    """Rows of W windows: most below twice the mean, some empty, a few long."""
    rng = np.random.default_rng(seed)
    lengths = rng.integers(0, 2 * mean, W)
    lengths[rng.integers(0, W, W // 12)] = 0
    lengths[rng.choice(W, len(longest), replace=False)] = longest
    return lengths.tolist()


# Waves across the channels and, in the gradients, workgroups there: with 32 or 64 groups as many of both, at
# 1,024 channels of one group 16 and 4 (at 4 states), at 256 channels of 16 groups 16 and 16.
@pytest.mark.parametrize("lengths,D,N,G,dtype,kw", [
    # 4,096 waves and more: parts of four times the mean, 72 to 136 rows here, of which some windows have several
    (uneven(130, 26, [600, 135, 136, 137, 272, 273], 1), 64, 16, 32, "f32", dict(state=True)),
    (uneven(130, 26, [600, 121, 300], 2), 64, 8, 32, "bf16", dict(state=True, order=True)),
    # parts of 512, the longest there are
    (uneven(130, 120, [1300, 512, 513, 511, 1024, 1025], 3), 64, 4, 32, "f32", dict(state=True, gate=False)),
    (uneven(260, 24, [400, 100, 101], 4), 1024, 4, 1, "f16", dict(strided=True)),
    (uneven(260, 20, [300, 64, 65, 129], 5), 256, 16, 16, "bf16", dict(state=True, front=3, behind=5)),
    # 64 states: the gradients' parts have 128 rows
    (uneven(130, 20, [500, 128, 129, 256, 257], 6), 64, 64, 32, "f32", dict(state=True)),
    # few windows, parts of 72, 112 and 128 rows
    ([6000, 0, 3999, 1], 64, 4, 64, "f32", dict(state=True)),
    ([14999], 64, 1, 64, "bf16", dict()),
    ([10000, 6601], 64, 4, 64, "f16", dict(state=True, order=True)),
    # few windows, the gradients' parts of 40, 56 and 64 rows
    ([1400, 101], 64, 16, 32, "f32", dict(state=True)),
    ([1999], 64, 12, 32, "bf16", dict(strided=True)),
    ([1290, 1000], 64, 32, 32, "f32", dict(state=True)),
])
def test_long_parts_and_many_windows(sla, lengths, D, N, G, dtype, kw):
    c = Case(lengths, D, N, dtype, G, seed=D + N, **kw)
    c.forward(sla)
    c.backward(sla, bar=1.5e-5 if N == 64 else 1e-5)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [1, 4, 8, 16, 32, 64])
def test_rows_alone(sla, dtype, N):
    """Neither gate nor skip, bias or softplus, in every type and at every number of states a lane is built for."""
    c = Case([90, 0, 3, 180], 70, N, dtype, seed=33, state=True, gate=False, skip=False, bias=False, softplus=False)
    c.forward(sla)
    c.backward(sla)
