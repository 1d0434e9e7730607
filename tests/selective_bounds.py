"""The selective scan in 64 bits, with how far a computation in 32 bits may be from it: an error carried along the recurrence, frame by frame (numpy; no code of the package).

h = 2^-24 is half a step of 32 bits.  To first order (all bounds times 1.01):

  step    r = softplus(s), s = dt + bias: s is off by h |s|, of which softplus keeps its slope, sigmoid(s) <= r; the exponential's argument by 1.5 h |s| (log2 e, and a product), the
          exponential by 2^-22 (approximate, or two units in the last place), and sums, a reciprocal (one unit), products and a polynomial by 7 h:  dr = 3 h |s| + 2^-20 of r.
          Without softplus: dr = h.
  decay   exp(r a): the exponent E = |r a| by dr, a in base 2 (1.5 h), a product (h), and where frames are carried over together a sum of up to 32 steps (31 h) and what segments add to it (h);
          the exponential by 2^-22:  dd = E (dr + 35 h) + 2^-22.
  state   what enters, r u b, by dr and two products (2 h); the sum by h, and by h again where a chunk's or segment's parts are joined.
  output  sum_n c h: states + 8 sums, d u and its sum 2 h; gate: 2^-22 of an exponential whose argument is off by 1.5 h |z|, a sum, a reciprocal and two products (5 h).
"""
from __future__ import annotations

import numpy as np

from tests.selective_oracle import sigmoid, softplus

H = 2.0 ** -24


def scan(u, dt, a, b, c, d=None, z=None, dt_bias=None, plus=True, state=None):
    """u, dt, z [T][B][C], a [C][N], b, c [T][B][G][N], state [B][C][N].  Returns out, its bound, the last states, their bound."""
    u, dt, a, b, c = (np.asarray(x, np.float64) for x in (u, dt, a, b, c))
    T, B, C = u.shape
    N = a.shape[1]
    share = C // b.shape[2]
    h = np.zeros((B, C, N)) if state is None else np.asarray(state, np.float64).copy()
    m, e = np.abs(h), np.zeros((B, C, N))
    out, bound = np.zeros((T, B, C)), np.zeros((T, B, C))
    for t in range(T):
        s = dt[t] + (0 if dt_bias is None else np.asarray(dt_bias, np.float64))
        r = softplus(s) if plus else s
        dr = (3 * H * np.abs(s) + 2.0 ** -20 if plus else np.full(s.shape, H))[..., None]
        bt, ct = np.repeat(b[t], share, axis=1), np.repeat(c[t], share, axis=1)
        exponent = r[..., None] * a
        decay, x = np.exp(exponent), (r * u[t])[..., None] * bt
        e = decay * (e + m * (np.abs(exponent) * (dr + 35 * H) + 2.0 ** -22)) + np.abs(x) * (dr + 2 * H)
        h, m = decay * h + x, decay * m + np.abs(x)
        e += 2 * H * m
        out[t], bound[t] = (ct * h).sum(-1), (np.abs(ct) * (e + (N + 10) * H * m)).sum(-1)
        mag = (np.abs(ct) * m).sum(-1)
        if d is not None:
            skip = np.asarray(d, np.float64) * u[t]
            out[t] += skip
            bound[t] += 2 * H * (mag + np.abs(skip))
            mag += np.abs(skip)
        if z is not None:
            gate = np.asarray(z[t], np.float64) * sigmoid(np.asarray(z[t], np.float64))
            out[t] *= gate
            bound[t] = np.abs(gate) * (bound[t] + mag * (2.0 ** -22 + 1.5 * H * np.abs(z[t]) + 5 * H))
    return out, 1.01 * bound + 1e-30, h, 1.01 * e + 1e-30
