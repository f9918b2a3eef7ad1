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
