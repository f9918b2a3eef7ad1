"""CPU tests of what a program relies on around the calls of the short convolution, the selective scan and the
residual normalisation: which buffers they refuse (before anything is launched), what workspaces are enough, and
first calls by several threads."""
from __future__ import annotations

import os

import pytest

from paper_2401_00912_amd import sla
from tests.test_space_cpu import CONV, CONV_BWD, CONV_FWD, CONV_STEP, FAKE, NORM, NORM_BWD, NORM_FWD, SCAN, SCAN_BWD, SCAN_FWD
from tests.test_space_cpu import SCAN_STEP, call

one, two = FAKE * 201, FAKE * 202   # addresses that nothing else has


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sla.LIB_PATH):
        from paper_2401_00912_amd import build

        build.build()
    return sla.lib()


def refused(f, names, defaults, outputs, inputs, allowed=(), **given):
    """Each pair of outputs and of an output and an input in one buffer, but the allowed ones, is refused."""
    defaults = dict(defaults, **given)
    assert len({defaults[k] for k in (*outputs, *inputs)}) == len(outputs) + len(inputs), "addresses that differ"
    for i, o in enumerate(outputs):
        for other in (*outputs[:i], *inputs):
            if (o, other) not in allowed:
                assert call(f, names, defaults, {o: defaults[other]}) == sla.SLA_E_ARG, (o, other)


# ------------------------------------------------------------------ one buffer for two things
def test_conv_outputs_apart(L):
    refused(L.sla_forward_short_conv, CONV_FWD, CONV, ("y", "so"), ("x", "w", "b", "s", "offsets", "order"), s=one, so=two,
            order=FAKE * 203)
    refused(L.sla_backward_short_conv, CONV_BWD, CONV, ("dx", "dw", "db", "dsi"),
            ("x", "w", "b", "s", "dy", "ds", "offsets", "order"), s=one, ds=two, dsi=FAKE * 203, order=FAKE * 204)
    refused(L.sla_step_short_conv, CONV_STEP, CONV, ("y", "pool"), ("x", "w", "b", "slots"))


def test_scan_outputs_apart(L):
    rows = ("x", "d", "A", "B", "C", "skip", "z", "bias")
    refused(L.sla_forward_selective_scan, SCAN_FWD, SCAN, ("y", "so"), (*rows, "s", "offsets", "order"), [("so", "s")], s=one,
            so=two, order=FAKE * 203)
    refused(L.sla_backward_selective_scan, SCAN_BWD, SCAN, ("dx", "dd", "dA", "dB", "dC", "dskip", "dz", "dbias", "dsi"),
            (*rows, "s", "dy", "ds", "offsets", "order"), [("dsi", "ds")], s=one, ds=two, dsi=FAKE * 203, order=FAKE * 204)
    refused(L.sla_step_selective_scan, SCAN_STEP, SCAN, ("y", "pool"), (*rows, "slots"))


def test_norm_outputs_apart(L):
    refused(L.sla_forward_residual_norm, NORM_FWD, NORM, ("y", "ro", "rstd", "ps"), ("x", "r", "g", "w", "pw"), [("ro", "r")])
    refused(L.sla_backward_residual_norm, NORM_BWD, NORM, ("dx", "dr", "dg", "dw", "dpw"),
            ("x", "ro", "g", "w", "pw", "rstd", "ps", "dy", "dro"), [("dr", "dro")])


def test_without_rows_only_the_parameters_count(L):
    """Tensors without rows have any address, the same one too: what is refused is for parameters and states alone."""
    for f, order, defaults, keys, same in (
            (L.sla_backward_short_conv, CONV_BWD, CONV, ("x", "dy", "dx"), dict(db=CONV["dw"])),
            (L.sla_backward_selective_scan, SCAN_BWD, SCAN, ("x", "d", "B", "C", "z", "dy", "dx", "dd", "dB", "dC", "dz"),
             dict(dbias=SCAN["dskip"])),
            (L.sla_backward_residual_norm, NORM_BWD, NORM, ("x", "ro", "g", "dy", "dro", "dx", "dr", "dg"),
             dict(dpw=NORM["dw"]))):
        # a workspace that is too small is refused after the addresses have been looked at
        empty = dict({k: one for k in keys}, n=0, nbytes=0)
        assert call(f, order, defaults, empty) == sla.SLA_E_WORKSPACE
        assert call(f, order, defaults, dict(empty, **same)) == sla.SLA_E_ARG


# ------------------------------------------------------------------ first calls by several threads
def test_a_first_call_beside_another_threads_first_call(monkeypatch):
    """A second thread whose first call falls into the first one's own finds every type."""
    import threading

    import torch

    found = []

    def second():
        try:
            found.extend(sla._dtype_code(t) for t in (torch.float32, torch.float16, torch.bfloat16))
        except TypeError as e:
            found.append(str(e))

    class Codes(dict):
        def update(self, *args):
            if threading.current_thread() is threading.main_thread():
                other = threading.Thread(target=second)
                other.start()
                other.join(30)
            super().update(*args)

    monkeypatch.setattr(sla, "_dtype_codes", Codes())
    monkeypatch.setattr(sla, "_torch_module", None)
    assert sla._dtype_code(torch.bfloat16) == 2
    assert found == [0, 1, 2]


# ------------------------------------------------------------------ workspaces
def test_a_workspace_is_enough_for_fewer_rows_and_windows(L):
    """Where strips and parts get longer, and at sizes all over the range."""
    import random

    conv = lambda n, W, dtype, D, N: L.sla_short_conv_backward_workspace_bytes(n, W, dtype, D, 4)  # noqa: E731
    forward = lambda n, W, dtype, D, N: L.sla_selective_scan_workspace_bytes(n, W, dtype, D, 1, N)  # noqa: E731
    back = lambda n, W, dtype, D, N: L.sla_selective_scan_backward_workspace_bytes(n, W, dtype, D, 1, N)  # noqa: E731
    norm = lambda n, W, dtype, D, N: L.sla_residual_norm_backward_workspace_bytes(n, dtype, D)  # noqa: E731
    assert conv(12223, 9, 2, 2048, 0) <= conv(16394, 9, 2, 2048, 0)
    assert forward(59837, 1023, 1, 256, 16) <= forward(59837, 1024, 1, 256, 16)
    assert back(10234, 2, 2, 1024, 1) <= back(10287, 2, 2, 1024, 1)
    rng = random.Random(11)
    size = lambda hi: int(hi ** rng.random())  # noqa: E731
    for _ in range(4000):
        dtype, D, N = rng.randrange(3), rng.choice([1, 70, 256, 1024, 2048, 8192]), rng.choice([1, 4, 8, 16, 32, 64])
        n, W = size(300000), size(5000)
        more_n, more_W = n + rng.choice([0, 1, 8, size(60000)]), W + rng.choice([0, 1, size(3000)])
        for f in (conv, forward, back, norm):
            assert 0 < f(n, W, dtype, D, N) <= f(more_n, more_W, dtype, D, N), (n, W, more_n, more_W, dtype, D, N)
