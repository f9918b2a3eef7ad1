"""Float64 references of the gated delta rule and of group normalisation, row by row from the
definitions (include/sla.h).  numpy only, independent of the library."""
from __future__ import annotations

import numpy as np


def _wide(x, heads):
    """One query/key head for each value head."""
    return np.repeat(np.asarray(x, np.float64), heads // x.shape[1], axis=1)


def _windows(offsets, order, n):
    rows = np.arange(n) if order is None else np.asarray(order, np.int64)
    return [rows[offsets[w]: offsets[w + 1]] for w in range(len(offsets) - 1)]


def delta_forward_ref(q, k, v, g, beta, offsets, scale, state=None, order=None):
    """(o [n, heads, dim_v], states [windows, heads, dim_k, dim_v]); rows in no window: NaN."""
    v, g, beta = (np.asarray(x, np.float64) for x in (v, g, beta))
    H = v.shape[1]
    q, k = _wide(q, H), _wide(k, H)
    o = np.full(v.shape, np.nan)
    W = len(offsets) - 1
    S = np.zeros((W, H, k.shape[2], v.shape[2])) if state is None else np.array(state, np.float64)
    for w, rows in enumerate(_windows(offsets, order, v.shape[0])):
        for r in rows:
            S[w] *= np.exp(g[r])[:, None, None]
            u = beta[r][:, None] * (v[r] - np.einsum("hk,hkv->hv", k[r], S[w]))
            S[w] += k[r][:, :, None] * u[:, None, :]
            o[r] = scale * np.einsum("hk,hkv->hv", q[r], S[w])
    return o, S


def delta_step_ref(state, slots, q, k, v, g, beta, scale):
    """(o, states): the rows of a slot in row order; padding rows' o is NaN."""
    S = np.array(state, np.float64)
    o = np.full(v.shape, np.nan)
    for b, s in enumerate(slots):
        if 0 <= s < S.shape[0]:
            one, st = delta_forward_ref(q[b:b + 1], k[b:b + 1], v[b:b + 1], g[b:b + 1], beta[b:b + 1], [0, 1], scale,
                                        S[s:s + 1])
            o[b], S[s] = one[0], st[0]
    return o, S


def delta_backward_ref(q, k, v, g, beta, offsets, dout, scale, state=None, dstate=None, order=None):
    """(dq, dk, dv, dg, dbeta, dstate_in) by the chain rule of one row, from the last row to the first."""
    v, g, beta, dout = (np.asarray(x, np.float64) for x in (v, g, beta, dout))
    n, H = v.shape[:2]
    Hk = q.shape[1]
    q, k = _wide(q, H), _wide(k, H)
    dq, dk, dv, dg, db = (np.full(x.shape, np.nan) for x in (q, k, v, g, beta))
    W = len(offsets) - 1
    zero = np.zeros((W, H, k.shape[2], v.shape[2]))
    S0 = zero if state is None else np.asarray(state, np.float64)
    D = zero.copy() if dstate is None else np.array(dstate, np.float64)
    for w, rows in enumerate(_windows(offsets, order, n)):
        S, decayed, errors, after = S0[w].copy(), [], [], []
        for r in rows:
            A = S * np.exp(g[r])[:, None, None]
            e = v[r] - np.einsum("hk,hkv->hv", k[r], A)
            S = A + k[r][:, :, None] * (beta[r][:, None] * e)[:, None, :]
            decayed.append(A)
            errors.append(e)
            after.append(S)
        for r, A, e, S in zip(rows[::-1], decayed[::-1], errors[::-1], after[::-1]):
            dq[r] = scale * np.einsum("hkv,hv->hk", S, dout[r])
            G = D[w] + scale * q[r][:, :, None] * dout[r][:, None, :]
            du = np.einsum("hk,hkv->hv", k[r], G)
            de = beta[r][:, None] * du
            db[r] = (du * e).sum(-1)
            dv[r] = de
            dk[r] = np.einsum("hkv,hv->hk", G, beta[r][:, None] * e) - np.einsum("hkv,hv->hk", A, de)
            G = G - k[r][:, :, None] * de[:, None, :]
            dg[r] = (G * A).sum((-1, -2))
            D[w] = G * np.exp(g[r])[:, None, None]
    shared = lambda x: x.reshape(n, Hk, H // Hk, -1).sum(2)  # noqa: E731
    return shared(dq), shared(dk), dv, dg, db, D


ACTIVATIONS = {"none": lambda z: z, "relu": lambda z: np.where(z > 0, z, np.where(np.isnan(z), z, 0.0)),
               "silu": lambda z: z / (1 + np.exp(-z))}


def _slope(activation, z):
    if activation == "none":
        return np.ones_like(z)
    if activation == "relu":
        return (z > 0).astype(np.float64)
    s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def _segments(n, offsets):
    return [(r, r + 1) for r in range(n)] if offsets is None else list(zip(offsets[:-1], offsets[1:]))


def group_norm_forward_ref(x, groups, weight=None, bias=None, offsets=None, eps=1e-5, activation="none"):
    """(y, mean, rstd); rows in no window: NaN; a window without rows has mean 0, rstd 1 / sqrt(eps)."""
    x = np.asarray(x, np.float64)
    n, C = x.shape
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    segs = _segments(n, offsets)
    y = np.full(x.shape, np.nan)
    mean, rstd = np.zeros((len(segs), groups)), np.full((len(segs), groups), eps ** -0.5)
    for s, (lo, hi) in enumerate(segs):
        if hi <= lo:
            continue
        X = x[lo:hi].reshape(hi - lo, groups, -1)
        mean[s] = X.mean((0, 2))
        rstd[s] = (X.var((0, 2)) + eps) ** -0.5
        hat = (X - mean[s][None, :, None]) * rstd[s][None, :, None]
        y[lo:hi] = ACTIVATIONS[activation](hat.reshape(hi - lo, C) * w + b)
    return y, mean, rstd


def group_norm_backward_ref(x, groups, dy, mean, rstd, weight=None, bias=None, offsets=None, activation="none"):
    """(dx, dweight, dbias) with the given statistics."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    n, C = x.shape
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    dx, dw, db = np.full(x.shape, np.nan), np.zeros(C), np.zeros(C)
    for s, (lo, hi) in enumerate(_segments(n, offsets)):
        if hi <= lo:
            continue
        m, r = (np.asarray(t, np.float64)[s][None, :, None] for t in (mean, rstd))
        hat = (x[lo:hi].reshape(hi - lo, groups, -1) - m) * r
        flat = hat.reshape(hi - lo, C)
        dz = dy[lo:hi] * _slope(activation, flat * w + b)
        dw += (dz * flat).sum(0)
        db += dz.sum(0)
        dh = (dz * w).reshape(hi - lo, groups, -1)
        dx[lo:hi] = (r * (dh - dh.mean((0, 2), keepdims=True) - hat * (dh * hat).mean((0, 2), keepdims=True))
                     ).reshape(hi - lo, C)
    return dx, dw, db
