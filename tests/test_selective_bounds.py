"""The bound of the selective scan's error holds for its recurrence in 32 bits, and does not for one that loses a few of them."""
import numpy as np
import pytest

from tests import selective_bounds


def bf16(x):
    w = np.asarray(x, np.float32).view(np.uint32)
    return ((w + 0x7FFF + ((w >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)


def recurrence(u, dt, a, b, c, d, z, bias, state, rounded):
    """In 32 bits; `rounded` goes over every decay."""
    u, dt, a, b, c, d, z, bias, h = (np.asarray(x, np.float32) for x in (u, dt, a, b, c, d, z, bias, state))
    out = np.zeros_like(u)
    share = u.shape[2] // b.shape[2]
    for t in range(u.shape[0]):
        s = dt[t] + bias
        r = np.maximum(s, 0) + np.log1p(np.exp(-np.abs(s)))
        bt, ct = np.repeat(b[t], share, axis=1), np.repeat(c[t], share, axis=1)
        h = rounded(np.exp(r[..., None] * a)) * h + (r * u[t])[..., None] * bt
        out[t] = ((ct * h).sum(-1, dtype=np.float32) + d * u[t]) * (z[t] / (1 + np.exp(-z[t])))
    return out, h


@pytest.mark.parametrize("T,C,N", [(600, 20, 16), (130, 33, 16), (333, 2, 128), (3, 40, 8)])
def test_bound_tells_32_bits_from_less(T, C, N):
    rng = np.random.default_rng(1)
    u, dt, z = (rng.standard_normal((T, 2, C)).astype(np.float32) for _ in range(3))
    b, c = (rng.standard_normal((T, 2, 1, N)).astype(np.float32) for _ in range(2))
    a = (-np.arange(1, N + 1) * np.exp(0.2 * rng.standard_normal((C, N)))).astype(np.float32)
    d, bias, state = (rng.standard_normal(s).astype(np.float32) for s in ((C,), (C,), (2, C, N)))
    bias -= 3
    want, e, left, es = selective_bounds.scan(u, dt, a, b, c, d, z, bias, True, state)
    out, h = recurrence(u, dt, a, b, c, d, z, bias, state, lambda x: x)
    assert (np.abs(out - want) <= e).all() and (np.abs(h - left) <= es).all()
    for rounded, share in ((bf16, 0.5), (lambda x: x * np.float32(1 + 2.0 ** -13), 0.2)):
        out, h = recurrence(u, dt, a, b, c, d, z, bias, state, rounded)
        assert (np.abs(h - left) > es).mean() > share and (np.abs(out - want) > e).mean() > 0.1
    assert np.median(es / np.maximum(np.abs(left), 1e-3)) < 1e-4
