"""The short convolution's and the selective scan's edges: orders that name no row and workspaces of just the bytes
that are needed, against the float64 reference.  Tolerances are those of the operators' own tests."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import space_ref
from tests.gpu_util import torch_dtype
from tests.test_gpu_conv import Case as ConvCase
from tests.test_gpu_conv import close, within
from tests.test_gpu_scan import Case

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
