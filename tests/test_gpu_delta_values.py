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


# ------------------------------------------------------------------ keys of many sizes
def close_rows(got, ref, dtype, name, rows, bar=FP32_BAR):
    """Rows of one kind held to the largest among them."""
    import torch

    close(got[torch.from_numpy(rows)], ref[rows], dtype, name, bar)


# windows of a chunk and some, and one that is cut into parts of 512 rows
SMALL_KEYS = [("f32", 1e-6), ("f32", 1e-9), ("f32", 1e-12), ("f32", 1e-30), ("bf16", 1e-6), ("bf16", 1e-9),
              ("bf16", 1e-12), ("bf16", 1e-30), ("f16", 1e-4), ("f16", 1e-6)]


def small_keys(dtype, x, lengths, **kw):
    """A few keys x times as long as the others, whose betas are as ever: they write x times as much."""
    c = Case(lengths, 1, 2, 32, 32, dtype, seed=31, **kw)
    few = np.zeros(c.n, bool)
    few[[3, 40, 63, 66, 90, c.n - 2]] = True
    k = c.k.float()
    k[few] *= x
    c.k = k.to(c.k.dtype)
    return c, few


@pytest.mark.parametrize("lengths", [[70, 64], [1100, 70]])
@pytest.mark.parametrize("dtype,x", SMALL_KEYS)
def test_forward_with_a_small_key(sla, dtype, x, lengths):
    c, _ = small_keys(dtype, x, lengths, state=lengths[0] > 100)
    o, st = c.forward(sla)
    ro, rs = c.forward_ref()
    close(o, ro, dtype, "o")
    close(st, rs, "f32", "state")


@pytest.mark.parametrize("lengths", [[70, 64], [1100, 70]])
@pytest.mark.parametrize("dtype,x", SMALL_KEYS)
def test_backward_with_a_small_key(sla, dtype, x, lengths):
    c, few = small_keys(dtype, x, lengths, grads=True)
    for name, got, ref in gradients(sla, c):
        close_rows(got, ref, out_type(c, name), name, ~few)


def mixed_keys(dtype, lengths, **kw):
    """Keys of three sizes with betas that make up for it (beta |k|^2 as with keys of 1), so that every row
    writes as much as any other; the sizes' rows."""
    import torch

    c = Case(lengths, 1, 2, 64, 32, dtype, seed=32, **kw)
    sizes = (1.0, 256.0 if dtype == "f16" else 2.0 ** 20, 1.0 / 16)
    size = torch.tensor(sizes)[torch.arange(c.n) % 3]
    c.k = (c.k.float() * size[:, None, None]).to(c.k.dtype)
    c.beta = c.beta / size[:, None].square()
    c.beta[7] = 0
    c.k[11] = 0
    return c, [np.flatnonzero(size.numpy() == s) for s in sizes]


@pytest.mark.parametrize("lengths", [[150, 64], [1100, 70]])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_forward_with_keys_of_many_sizes(sla, dtype, lengths):
    c, _ = mixed_keys(dtype, lengths, state=True)
    o, st = c.forward(sla)
    ro, rs = c.forward_ref()
    close(o, ro, dtype, "o")
    close(st, rs, "f32", "state")


def test_betas_of_zero(sla):
    """Nothing is written, in a chunk or in a whole window: what is read and the betas' own gradients are as good
    as ever."""
    c = Case([200, 70], 1, 2, 32, 32, "f32", seed=33, state=True, grads=True)
    c.beta[64:128] = 0
    c.beta[200:] = 0
    o, st = c.forward(sla)
    ro, rs = c.forward_ref()
    close(o, ro, "f32", "o")
    close(st, rs, "f32", "state")
    for name, got, ref in gradients(sla, c):
        close(got, ref, "f32", name)


@pytest.mark.parametrize("lengths", [[70, 64], [1100, 70]])
@pytest.mark.parametrize("dtype,x", SMALL_KEYS)
def test_gradients_of_a_small_key(sla, dtype, x, lengths):
    """dk of the few small keys, which is as large as the others', and their dv and dbeta, which are x times as
    large (keys are scaled up to 2^60 times: at 1e-30 those two are not worth a bit beside the others)."""
    c, few = small_keys(dtype, x, lengths, grads=True)
    for name, got, ref in gradients(sla, c):
        if name == "dk" or (name in ("dv", "dbeta") and x > 1e-30 and dtype != "f16"):
            close_rows(got, ref, out_type(c, name), name, few)


@pytest.mark.parametrize("lengths", [[150, 64], [1100, 70]])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradients_with_keys_of_many_sizes(sla, dtype, lengths):
    """Each size's rows by themselves: dk is smaller and dbeta larger the larger a key is.  fp16's dk has steps of
    2^-24 whatever its size, and the row without a key has no size."""
    c, kinds = mixed_keys(dtype, lengths, state=True, grads=True)
    for name, got, ref in gradients(sla, c):
        if name == "dstate_in":
            close(got, ref, "f32", name)
            continue
        for rows in kinds:
            close_rows(got, ref, out_type(c, name), name, np.setdiff1d(rows, [11]))


# ------------------------------------------------------------------ parts that forget
@pytest.mark.parametrize("dk,dv", [(32, 32), (48, 64), (128, 16)])
def test_parts_that_forget_keep_their_bits(sla, dk, dv):
    """A window cut into parts of 512 rows, across each of which the state falls to e^-15 of itself and nothing is
    written: what is left of the state, its reads on the way and the gradient that comes back are as good, for
    their own size, as at the start."""
    import torch

    n, gam = 2100, -0.03
    c = Case([n], 1, 1, dk, dv, "f32", seed=35, state=True, grads=True)
    c.g[:] = gam
    c.beta[:] = 0
    c.dout[:] = 0
    o, st = c.forward(sla)
    ro, rs = c.forward_ref()
    up = np.exp(-gam * np.arange(1, n + 1))[:, None, None]
    close(o.double().cpu() * torch.from_numpy(up), ro * up, "f32", "o")
    close(st, rs, "f32", "state")
    for name, got, ref in gradients(sla, c):
        if name == "dstate_in":
            close(got, ref, "f32", name)
        if name == "dbeta":
            down = up[::-1, :, 0].copy()
            close(got.double().cpu() * torch.from_numpy(down), ref * down, "f32", name)


# ------------------------------------------------------------------ states that grow
@pytest.mark.parametrize("lengths,g", [([150, 70], 0.1), ([1100, 70], 0.02)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_states_that_grow(sla, dtype, lengths, g):
    """Log decays above zero: nothing overflows before the results do.  A chunk's products are up to e^(64 g) times
    the results that they cancel to, and so is the limit."""
    c = Case(lengths, 1, 2, 32, 32, dtype, seed=37, state=True, grads=True)
    c.g[:] = g
    # keys and queries of length 1 that have much in common, betas that write little of it off
    c.q, c.k = (((1 + x.float()) / (1 + x.float()).norm(dim=-1, keepdim=True)).to(x.dtype) for x in (c.q, c.k))
    c.beta /= 16
    c.v, c.dout = ((x.float() * 2.0 ** -12).to(x.dtype) for x in (c.v, c.dout))
    c.state, c.dstate = c.state * 2.0 ** -12, c.dstate * 2.0 ** -12
    if dtype == "f16" and g < 0.1:
        c.q /= 2.0 ** 14   # its results end at 65,504
        c.dout /= 2.0 ** 10
    bar = FP32_BAR * float(np.exp(64 * g))
    o, st = c.forward(sla)
    ro, rs = c.forward_ref()
    close(o, ro, dtype, "o", bar)
    close(st, rs, "f32", "state", bar)
    for name, got, ref in gradients(sla, c):
        close(got, ref, out_type(c, name), name, bar)


# ------------------------------------------------------------------ rows of many sizes
@pytest.mark.parametrize("lengths", [[150, 70], [1700, 70]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_before_a_large_one(sla, dtype, lengths):
    """A row's value 10^9 times the others': what came before it is as good as without it, and so are the gradients
    of what comes behind such a row of dout.  (Its chunk's other rows have 22 bits down to 2^-27 of it, and 19 at
    10^-9: a step of 2^-49 of it is 2e-6 of them.)"""
    at = 60
    c = Case(lengths, 1, 2, 64, 32, dtype, seed=38, grads=True)
    c.v[at] *= 1e9
    c.dout[at] *= 1e9
    o, _ = c.forward(sla)
    before = np.arange(c.n) < at
    close_rows(o, c.forward_ref()[0], dtype, "o", before)
    for name, got, ref in gradients(sla, c):
        if name == "dv":
            close_rows(got, ref, dtype, name, np.arange(c.n) > at)


# ------------------------------------------------------------------ columns of many sizes
def close_columns(got, ref, dtype, name):
    """Every head's columns, each held to its own largest."""
    for h in range(ref.shape[1]):
        for j in range(ref.shape[-1]):
            close(got[:, h, ..., j], ref[:, h, ..., j], dtype, f"{name} of head {h}, column {j}")


@pytest.mark.parametrize("lengths", [[150, 0, 64], [1700, 70]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 80), (128, 48)])
def test_columns_of_many_sizes(sla, dk, dv, dtype, lengths):
    """Value columns do not mix: columns 10^10 times as large or as small as their neighbours, in v, the states,
    dout and their gradients, each as good as alone."""
    c = Case(lengths, 1, 2, dk, dv, dtype, seed=34, state=True, grads=True)
    for x in (c.v, c.dout):
        x[:, 0, 5] *= 1e10
        x[:, 0, 17] *= 1e-10
        x[:, 1, 6] *= 1e5
    for x in (c.state, c.dstate):
        x[:, 0, :, 5] *= 1e10
        x[:, 0, :, 17] *= 1e-10
        x[:, 1, :, 9] *= 1e10
    o, st = c.forward(sla)
    ro, rs = c.forward_ref()
    close_columns(o, ro, dtype, "o")
    close_columns(st, rs, "f32", "state")
    for name, got, ref in gradients(sla, c):
        if name in ("dv", "dstate_in"):
            close_columns(got, ref, out_type(c, name), name)


# ------------------------------------------------------------------ gradients of fast decays
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("g", [-1.0, -8.0, -20.0])
def test_gradients_of_fast_decays(sla, dtype, g):
    """Heads that forget fast all along: dg is e^g times what it is summed from, and is held to the bound that the
    interface gives, 1e-5 of the head's own largest |o| |dout| + |v| |dv|, and to nothing of another head."""
    import torch

    c = Case([300, 70], 1, 2, 64, 64, dtype, seed=40, state=True, grads=True)
    c.g[:, 0] = g
    c.g[:, 1] = g * (0.5 + torch.rand(c.n, generator=torch.Generator().manual_seed(1)))
    c.dout[:, 1] /= 1024
    c.dstate[:, 1] /= 1024
    ref = {name: (got.double().cpu().numpy(), want) for name, got, want in gradients(sla, c)}
    norm = lambda x: np.sqrt((x ** 2).sum(-1))  # noqa: E731
    bound = norm(c.forward_ref()[0]) * norm(c.wide("dout")) + norm(c.wide("v")) * norm(ref["dv"][1])
    worst = np.abs(ref["dg"][0] - ref["dg"][1]).max(0) / (FP32_BAR * bound.max(0))
    assert (worst <= 1).all(), worst
