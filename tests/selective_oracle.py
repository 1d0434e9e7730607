"""The operators of the selective head in 64 bits, as they are defined, with the magnitudes that error bounds need (numpy; no code of the package)."""
from __future__ import annotations

import numpy as np

HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-x))


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def conv(x, weight, bias=None, silu=False, state=None):
    """One sequence: x [T][C], weight [C][W], state [W - 1][C].  Returns out, the last W - 1 frames, and the sums ahead of the activation with their terms' magnitudes."""
    x, weight = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    T, C = x.shape
    W = weight.shape[1]
    seen = np.concatenate((np.zeros((W - 1, C)) if state is None else np.asarray(state, np.float64), x))
    y = np.zeros((T, C)) if bias is None else np.broadcast_to(np.asarray(bias, np.float64), (T, C)).copy()
    mag = np.abs(y)
    for j in range(W):
        y += weight[:, j] * seen[j:j + T]
        mag += np.abs(weight[:, j] * seen[j:j + T])
    return (y * sigmoid(y) if silu else y), seen[seen.shape[0] - (W - 1):], mag


def scan(u, dt, a, b, c, d=None, z=None, dt_bias=None, plus=True, state=None):
    """One sequence: u, dt, z [T][C], a [C][N], b, c [T][G][N], state [C][N].  Returns out, the last state, every term's magnitude in the place of both, and the largest
    exponent of a decay."""
    u, dt, a, b, c = (np.asarray(x, np.float64) for x in (u, dt, a, b, c))
    T, C = u.shape
    N = a.shape[1]
    share = C // b.shape[1]
    h = np.zeros((C, N)) if state is None else np.asarray(state, np.float64).copy()
    m = np.abs(h)
    out, mag, top = np.zeros((T, C)), np.zeros((T, C)), 0.0
    for t in range(T):
        r = dt[t] + (0 if dt_bias is None else np.asarray(dt_bias, np.float64))
        r = softplus(r) if plus else r
        bt, ct = np.repeat(b[t], share, axis=0), np.repeat(c[t], share, axis=0)
        decay = np.exp(r[:, None] * a)
        top = max(top, float(np.abs(r[:, None] * a).max()))
        h = decay * h + (r * u[t])[:, None] * bt
        m = decay * m + np.abs((r * u[t])[:, None] * bt)
        out[t], mag[t] = (ct * h).sum(-1), (np.abs(ct) * m).sum(-1)
        if d is not None:
            out[t] += np.asarray(d, np.float64) * u[t]
            mag[t] += np.abs(np.asarray(d, np.float64) * u[t])
    if z is not None:
        gate = np.asarray(z, np.float64) * sigmoid(np.asarray(z, np.float64))
        out, mag = out * gate, mag * np.abs(gate)
    return out, h, mag, m, top


def scan_error(frames, states, top):
    """Largest error of a sum, over the sum of its terms' magnitudes: per frame a decay (2^-22 of an approximate exponential, and its exponent times 2^-21: two roundings of the
    step ahead of the softplus and in it, one of the product and one of a in base 2), then the readout's products, sums, gate."""
    return (frames + 1) * (2.0 ** -22 + min(top, 100.0) * 2.0 ** -21) + (states + 16) * 2.0 ** -23 + 2.0 ** -19


def rms(x, weight, eps):
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if weight is None else y * np.asarray(weight, np.float64)


def block(y, residual, after=None, before=None, gate=None, act="sigmoid", scale=1.0, eps=1e-6, norms="both"):
    """Returns out (or None), h, and the magnitudes of h's two terms."""
    y, residual = np.asarray(y, np.float64), np.asarray(residual, np.float64)
    p = rms(y, after, eps) if norms in ("both", "after") else y
    if gate is not None:
        g = np.asarray(gate, np.float64)
        p = p * (g if act == "none" else sigmoid(g) if act == "sigmoid" else g * sigmoid(g))
    h = residual + scale * p
    mag = np.abs(residual) + np.abs(scale * p)
    return (rms(h, before, eps) if norms in ("both", "before") else None), h, mag
