"""The gated delta rule on values that share a tile with others far from their size: each column,
row and head is held to its own size, and not to the largest value beside it.

Tolerances.  As in the operator's other tests an fp32 result is off by at most 1e-5 of the largest
result (ten operands in two fp16 terms, each off by 2^-22 of what it is summed with, times 4 for
differences of larger terms), and a 16-bit result by half a step of its value more.  Here "the
largest" is taken over what may share a scale: one column of one head, or the rows of one kind."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import delta_ref
from tests.test_gpu_delta import FP32_BAR, GRADS, HALF_STEP, Case, close

pytestmark = pytest.mark.gpu

ROWS = ("q", "k", "v", "g", "beta")


@pytest.fixture(scope="module")
def sla():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2401_00912_amd import sla as S

    S.lib()
    return S


def gradients(S, c):
    """(name, kernel's, reference) of every gradient."""
    got = S.backward_delta(*(c.dev(x) for x in (*ROWS, "offsets", "dout")), dstate=c.dev("dstate"), order=c.dev("order"),
                           state=c.dev("state"))
    ref = delta_ref.delta_backward_ref(*(c.wide(x) for x in ROWS), c.offsets, c.wide("dout"), c.scale, c.wide("state"),
                                       c.wide("dstate"), c.wide("order"))
    return [(n, x, r) for n, x, r in zip(GRADS, got, ref) if x is not None]


def out_type(c, name):
    return c.dtype if name in ("o", "dq", "dk", "dv") else "f32"


# ------------------------------------------------------------------ bf16 rows
@pytest.mark.parametrize("lengths", [[150, 7, 64], [1100, 70]])
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 2, 32, 48), (2, 2, 64, 64), (1, 2, 128, 128)])
def test_bf16_results_are_rounded_once(sla, hk, h, dk, dv, lengths):
    """o, dq and dk of bf16 rows are as good as an fp32 result rounded once, however small beside the
    largest: their operands have as many bits as those of every other type."""
    c = Case(lengths, hk, h, dk, dv, "bf16", seed=dk, state=True, grads=True)
    o, _ = c.forward(sla)
    close(o, c.forward_ref()[0], "bf16", "o")
    for name, got, ref in gradients(sla, c):
        close(got, ref, out_type(c, name), name)
