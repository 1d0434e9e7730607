"""The operators of the temporal head in 64 bits, as they are defined, with the sums of magnitudes that error bounds need (numpy; no code of the
package)."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])   # 127 is NaN
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "mx8": 2.0 ** -4}


def nearest(table, a):
    """Codes of the entries nearest to a >= 0, ties to the even code."""
    hi = np.clip(np.searchsorted(table, a), 1, len(table) - 1)
    lo = hi - 1
    below, above = a - table[lo], table[hi] - a
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def quantize(x, fmt):
    """(codes [rows][groups * 32], scale bytes [rows][groups], values [rows][cols]) of x [rows][cols]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    groups = -(-cols // 32)
    y = np.zeros((rows, groups * 32))
    y[:, :cols] = x
    y = y.reshape(rows, groups, 32)
    table, top = (E2M1, 6.0) if fmt == "mx4" else (E4M3, 448.0)
    bad = ~np.isfinite(y).all(-1)
    most = np.where(bad, 0.0, np.abs(np.where(np.isfinite(y), y, 0.0)).max(-1))
    k = np.full(most.shape, -127)
    for i in np.ndindex(most.shape):
        while most[i] > top * 2.0 ** k[i]:
            k[i] += 1
    z = np.where(bad[..., None], 0.0, np.where(np.isfinite(y), y, 0.0) / 2.0 ** k[..., None].astype(np.float64))
    code = nearest(table, np.abs(z))
    values = np.where(np.signbit(z), -1, 1) * table[code] * 2.0 ** k[..., None].astype(np.float64)
    values = np.where(bad[..., None], np.nan, values)
    code = code + np.where(np.signbit(z), 8 if fmt == "mx4" else 128, 0)
    return code.reshape(rows, -1), np.where(bad, 255, k + 127), values.reshape(rows, -1)[:, :cols]


def pack(code, scales, fmt):
    """(data, scales) as they lie in memory; scale bytes of rows behind the last one are 0 here."""
    rows, groups = scales.shape
    data = (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8) if fmt == "mx4" else code.astype(np.uint8)
    tr, tg = -(-rows // 128), -(-groups // 4)
    s = np.zeros(tr * tg * 512, np.uint8)
    for r in range(rows):
        for g in range(groups):
            s[(r // 128 * tg + g // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + g % 4] = scales[r, g]
    return data, s


def norm(x, weight=None, residual=None, eps=1e-6):
    x = np.asarray(x, np.float64)
    s = x if residual is None else x + np.asarray(residual, np.float64)
    y = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    return (y if weight is None else y * np.asarray(weight, np.float64)), s


def attention(q, k, v, log_decay, state=None, scale=1.0):
    """One sequence: q [T][H][dk], k [T][G][dk], v [T][G][dv], log_decay [G] or [T][G], state [G][dk][dv].
    Returns out [T][H][dv], last state, and both with every term's magnitude in its place."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, H, dk = q.shape
    G, dv = v.shape[1:]
    with np.errstate(under="ignore"):
        d = np.exp(np.broadcast_to(np.asarray(log_decay, np.float64), (T, G)))
    S = np.zeros((G, dk, dv)) if state is None else np.asarray(state, np.float64).copy()
    A = np.abs(S)
    out, mag = np.zeros((T, H, dv)), np.zeros((T, H, dv))
    for t in range(T):
        S = d[t][:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
        A = d[t][:, None, None] * A + np.abs(k[t])[:, :, None] * np.abs(v[t])[:, None, :]
        out[t] = scale * np.einsum("ghi,gij->ghj", q[t].reshape(G, H // G, dk), S).reshape(H, dv)
        mag[t] = abs(scale) * np.einsum("ghi,gij->ghj", np.abs(q[t]).reshape(G, H // G, dk), A).reshape(H, dv)
    return out, S, mag, A
