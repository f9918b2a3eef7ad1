"""Float64 references of the short causal convolution, the selective scan and the residual
normalisation, row by row from the definitions (include/sla.h).  numpy only, independent of the
library."""
from __future__ import annotations

import numpy as np


def _windows(offsets, order, n):
    rows = np.arange(n) if order is None else np.asarray(order, np.int64)
    return [rows[offsets[w]: offsets[w + 1]] for w in range(len(offsets) - 1)]


def _sigmoid(z):
    return np.exp(-np.logaddexp(0.0, -z))


def _act(name, z):
    return z if name == "none" else np.maximum(z, 0.0) if name == "relu" else z * _sigmoid(z)


def _slope(name, z):
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return (z > 0).astype(np.float64)
    s = _sigmoid(z)
    return s * (1 + z * (1 - s))


# ------------------------------------------------------------------ short convolution
def conv_forward_ref(x, weight, offsets, bias=None, activation="none", order=None, state=None):
    """(y, states [windows, width - 1, channels]); rows in no window: NaN."""
    x, weight = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    n, C = x.shape
    K = weight.shape[1]
    y = np.full(x.shape, np.nan)
    W = len(offsets) - 1
    out = np.zeros((W, K - 1, C)) if state is None else np.array(state, np.float64)
    for w, rows in enumerate(_windows(offsets, order, n)):
        for r in rows:
            seen = np.concatenate([out[w], x[r][None]])
            z = (seen * weight.T).sum(0) + (0.0 if bias is None else bias)
            y[r] = _act(activation, z)
            out[w] = seen[1:]
    return y, out


def conv_backward_ref(x, weight, offsets, dy, bias=None, activation="none", order=None, state=None, dstate=None):
    """(dx, dweight, dbias, dstate_in); rows in no window: NaN."""
    x, weight, dy = (np.asarray(t, np.float64) for t in (x, weight, dy))
    n, C = x.shape
    K = weight.shape[1]
    dx, dw, db = np.full(x.shape, np.nan), np.zeros_like(weight), np.zeros(C)
    W = len(offsets) - 1
    start = np.zeros((W, K - 1, C)) if state is None else np.asarray(state, np.float64)
    back = np.zeros((W, K - 1, C)) if dstate is None else np.array(dstate, np.float64)
    for w, rows in enumerate(_windows(offsets, order, n)):
        full = np.concatenate([start[w], x[rows]])
        d = np.zeros_like(full)
        d[len(rows):] += back[w]
        for t, r in enumerate(rows):
            z = (full[t:t + K] * weight.T).sum(0) + (0.0 if bias is None else bias)
            dz = dy[r] * _slope(activation, z)
            d[t:t + K] += dz * weight.T
            dw += (dz * full[t:t + K]).T
            db += dz
        dx[rows] = d[K - 1:]
        back[w] = d[:K - 1]
    return dx, dw, db, back


def conv_step_ref(state, slots, x, weight, bias=None, activation="none"):
    """(y, states): the rows of a slot in row order; padding rows' y is NaN."""
    S = np.array(state, np.float64)
    y = np.full(x.shape, np.nan)
    for b, s in enumerate(slots):
        if 0 <= s < S.shape[0]:
            one, st = conv_forward_ref(x[b:b + 1], weight, [0, 1], bias, activation, state=S[s:s + 1])
            y[b], S[s] = one[0], st[0]
    return y, S


# ------------------------------------------------------------------ selective scan
def _scan_rows(x, delta, A, B, C, skip, z, delta_bias, softplus):
    x, delta, A = (np.asarray(t, np.float64) for t in (x, delta, A))
    D, G = x.shape[1], B.shape[1]
    B, C = (np.repeat(np.asarray(t, np.float64), D // G, axis=1) for t in (B, C))
    pre = delta + (0.0 if delta_bias is None else delta_bias)
    dt = np.logaddexp(0.0, pre) if softplus else pre
    return x, pre, dt, A, B, C, np.zeros(D) if skip is None else np.asarray(skip, np.float64)


def scan_forward_ref(x, delta, A, B, C, offsets, skip=None, z=None, delta_bias=None, delta_softplus=False, order=None,
                     state=None):
    """(y, states [windows, channels, states]); rows in no window: NaN."""
    x, _, dt, A, B, C, skip = _scan_rows(x, delta, A, B, C, skip, z, delta_bias, delta_softplus)
    W = len(offsets) - 1
    h = np.zeros((W, *A.shape)) if state is None else np.array(state, np.float64)
    y = np.full(x.shape, np.nan)
    for w, rows in enumerate(_windows(offsets, order, x.shape[0])):
        for r in rows:
            h[w] = np.exp(dt[r][:, None] * A) * h[w] + (dt[r] * x[r])[:, None] * B[r]
            y[r] = (C[r] * h[w]).sum(-1) + skip * x[r]
    return (y if z is None else y * _act("silu", np.asarray(z, np.float64))), h


def scan_backward_ref(x, delta, A, B, C, offsets, dy, skip=None, z=None, delta_bias=None, delta_softplus=False, order=None,
                      state=None, dstate=None):
    """(dx, ddelta, dA, dB, dC, dskip, dz, ddelta_bias, dstate_in) by the chain rule of one row, from the last row
    to the first; rows in no window: NaN."""
    G = B.shape[1]
    x, pre, dt, A, B, C, skip = _scan_rows(x, delta, A, B, C, skip, z, delta_bias, delta_softplus)
    n, D = x.shape
    N = A.shape[1]
    dy = np.asarray(dy, np.float64)
    W = len(offsets) - 1
    h0 = np.zeros((W, D, N)) if state is None else np.asarray(state, np.float64)
    back = np.zeros((W, D, N)) if dstate is None else np.array(dstate, np.float64)
    dx, dd, dz = (np.full(x.shape, np.nan) for _ in range(3))
    dB, dC = (np.full((n, G, N), np.nan) for _ in range(2))
    dA, dskip, dbias = np.zeros_like(A), np.zeros(D), np.zeros(D)
    shared = lambda t: t.reshape(G, D // G, N).sum(1)  # noqa: E731
    for w, rows in enumerate(_windows(offsets, order, n)):
        h, kept = h0[w], []
        for r in rows:
            a = np.exp(dt[r][:, None] * A) * h
            h = a + (dt[r] * x[r])[:, None] * B[r]
            kept.append((a, h))
        for r, (a, h) in zip(rows[::-1], kept[::-1]):
            g = dy[r]
            if z is not None:
                dz[r] = g * ((C[r] * h).sum(-1) + skip * x[r]) * _slope("silu", np.asarray(z[r], np.float64))
                g = g * _act("silu", np.asarray(z[r], np.float64))
            q = back[w] + g[:, None] * C[r]
            dC[r] = shared(g[:, None] * h)
            dB[r] = shared(q * (dt[r] * x[r])[:, None])
            du = (q * B[r]).sum(-1)
            dx[r] = du * dt[r] + g * skip
            ddt = du * x[r] + (q * a * A).sum(-1)
            dd[r] = ddt * (_sigmoid(pre[r]) if delta_softplus else 1.0)
            dA += q * a * dt[r][:, None]
            dskip += g * x[r]
            dbias += dd[r]
            back[w] = q * np.exp(dt[r][:, None] * A)
    return dx, dd, dA, dB, dC, dskip, dz, dbias, back


def scan_step_ref(state, slots, x, delta, A, B, C, skip=None, z=None, delta_bias=None, delta_softplus=False):
    """(y, states): the rows of a slot in row order; padding rows' y is NaN."""
    S = np.array(state, np.float64)
    y = np.full(x.shape, np.nan)
    for b, s in enumerate(slots):
        if 0 <= s < S.shape[0]:
            one = slice(b, b + 1)
            out, st = scan_forward_ref(x[one], delta[one], A, B[one], C[one], [0, 1], skip, None if z is None else z[one],
                                       delta_bias, delta_softplus, state=S[s:s + 1])
            y[b], S[s] = out[0], st[0]
    return y, S


# ------------------------------------------------------------------ residual normalisation
def rnorm_forward_ref(x, residual, weight=None, post_weight=None, gate=None, activation="none", scale=1.0, eps=1e-5):
    """(y, residual_out, rstd, post_rstd)"""
    u = np.asarray(x, np.float64)
    post = None
    if post_weight is not None:
        post = 1 / np.sqrt((u * u).mean(-1) + eps)
        u = u * post[:, None] * post_weight
    if gate is not None:
        u = u * _act(activation, np.asarray(gate, np.float64))
    r = scale * u + (0.0 if residual is None else np.asarray(residual, np.float64))
    rstd = 1 / np.sqrt((r * r).mean(-1) + eps)
    return r * rstd[:, None] * (1.0 if weight is None else weight), r, rstd, post


def rnorm_backward_ref(x, residual_out, dy, rstd, weight=None, post_weight=None, post_rstd=None, gate=None,
                       activation="none", scale=1.0, dresidual_out=None):
    """(dx, dresidual, dweight, dpost_weight, dgate)"""
    x, r, dy = (np.asarray(t, np.float64) for t in (x, residual_out, dy))

    def norm(v, s, d):
        hat = v * s[:, None]
        return s[:, None] * (d - hat * (d * hat).mean(-1, keepdims=True)), hat

    dr, hat = norm(r, rstd, dy if weight is None else dy * weight)
    dweight = (dy * hat).sum(0)
    if dresidual_out is not None:
        dr = dr + dresidual_out
    d = scale * dr
    u = x if post_weight is None else x * post_rstd[:, None] * post_weight
    dgate = None
    if gate is not None:
        gate = np.asarray(gate, np.float64)
        dgate = d * u * _slope(activation, gate)
        d = d * _act(activation, gate)
    dpost = None
    if post_weight is not None:
        dpost = (d * x * post_rstd[:, None]).sum(0)
        d, _ = norm(x, post_rstd, d * post_weight)
    return d, dr, dweight, dpost, dgate
