"""The short convolution's and the selective scan's edges: orders that name no row, and the sizes at which a call
goes another way (two channels a lane in single rows, long parts, many windows), against the float64 reference.
Tolerances are those of the operators' own tests."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import space_ref
from tests.gpu_util import torch_dtype
from tests.test_gpu_conv import Case as ConvCase
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


# ------------------------------------------------------------------ short convolution
@pytest.mark.parametrize("dtype,C,K", [("f32", 24, 4), ("bf16", 9, 8), ("f16", 64, 2)])
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
