"""Refusals, sizes and argument checks of the temporal head's operators: nothing here reaches a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import SrError, operators as ops
from tests import operator_oracle as oracle

INVALID, UNSUPPORTED = 1, 5
P = ctypes.c_void_p(1 << 20)                      # never read: every call here is refused, or has nothing to do
P2 = ctypes.c_void_p(1 << 21)


def desc(dtype=1, batch=2, heads=4, groups=2, dk=64, dv=64, frames=8, **strides):
    d = ops._AttentionDesc(dtype, batch, heads, groups, dk, dv, frames, 1.0)
    for name in ("q", "k", "v", "out", "log_decay"):
        setattr(d, name, ops._Strides(*strides.get(name, (batch * heads * 64, heads * 64, 64))))
    return d


def run(d, q=P, k=P, v=P, decay=P, offsets=None, s_in=None, s_out=None, out=P2, ws=None, size=0):
    return ops._library().sr_linear_attention_run(ctypes.byref(d) if d else None, q, k, v, decay, offsets, s_in, s_out, out, ws, size, None)


def step(d, q=P, k=P, v=P, decay=P, state=P, out=P2):
    return ops._library().sr_linear_attention_step(ctypes.byref(d) if d else None, q, k, v, decay, state, out, None)


@pytest.mark.parametrize("call", [run, step])
def test_attention_refuses_sizes_and_pointers(call):
    assert call(None) == INVALID
    for bad in (dict(dtype=2), dict(batch=-1), dict(heads=0), dict(groups=0), dict(heads=5), dict(dk=0), dict(dv=0), dict(frames=-1),
                dict(q=(-1, 1, 1)), dict(out=(1, -1, 1)), dict(log_decay=(0, 0, -1)), dict(batch=1 << 30, groups=4)):
        assert call(desc(**bad)) == INVALID, bad
    for bad in (dict(dk=257), dict(heads=129, groups=1)):
        assert call(desc(**bad)) == UNSUPPORTED, bad
    for name in ("q", "k", "v", "decay", "out"):
        assert call(desc(), **{name: None}) == INVALID, name
        assert call(desc(), **{name: ctypes.c_void_p((1 << 20) + 1)}) == INVALID, name
    for name in ("q", "k", "v"):
        assert call(desc(), **{name: P2}) == INVALID, name            # the outputs would lie on them
    assert call(desc(batch=0)) == 0


def test_attention_refuses_misaligned_states_and_a_short_workspace():
    odd = ctypes.c_void_p((1 << 20) + 2)
    assert run(desc(), s_in=odd) == INVALID and run(desc(), s_out=odd) == INVALID and run(desc(), offsets=odd) == INVALID
    assert step(desc(), state=odd) == INVALID and step(desc(), state=None) == INVALID
    size = ctypes.c_size_t()
    lib = ops._library()
    assert lib.sr_linear_attention_workspace_bytes(ctypes.byref(desc()), 0, None) == INVALID
    assert lib.sr_linear_attention_workspace_bytes(ctypes.byref(desc(dk=300)), 0, ctypes.byref(size)) == UNSUPPORTED
    assert lib.sr_linear_attention_workspace_bytes(ctypes.byref(desc(batch=1, heads=2, frames=1 << 16)), 0, ctypes.byref(size)) == 0
    if size.value:
        d = desc(batch=1, heads=2, frames=1 << 16)
        assert run(d, ws=ctypes.c_void_p(1 << 20), size=size.value - 1) == INVALID
        assert run(d, ws=None, size=size.value) == INVALID
        assert run(d, ws=ctypes.c_void_p((1 << 20) + 64), size=size.value) == INVALID


def test_microscale_refuses():
    lib = ops._library()
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    for rows, cols, fmt in ((-1, 32, 3), (4, 0, 3), (4, 32, 1), (4, 32, 4), (1 << 31, 32, 3), (4, 1 << 31, 3)):
        assert lib.sr_microscale_bytes(rows, cols, fmt, ctypes.byref(a), ctypes.byref(b)) == INVALID
    assert lib.sr_microscale_bytes(4, 32, 3, None, ctypes.byref(b)) == INVALID
    odd = ctypes.c_void_p((1 << 20) + 8)

    def quant(x=P, dtype=1, rows=4, cols=64, stride=64, fmt=3, data=P, scales=P):
        return lib.sr_microscale_quantize(x, dtype, rows, cols, stride, fmt, data, scales, None)
    for bad in (dict(x=None), dict(dtype=2), dict(rows=-1), dict(cols=0), dict(stride=-1), dict(fmt=0), dict(data=odd), dict(scales=odd), dict(data=None),
                dict(x=ctypes.c_void_p((1 << 20) + 1))):
        assert quant(**bad) == INVALID, bad
    assert quant(rows=0, x=None) == 0

    def prod(ad=P, asc=P, wd=P, wsc=P, fmt=3, rows=4, cols=64, outs=8, bias=None, act=0, out=P, dtype=1, stride=8):
        return lib.sr_microscale_product(ad, asc, wd, wsc, fmt, rows, cols, outs, bias, act, out, dtype, stride, None)
    for bad in (dict(ad=None), dict(asc=odd), dict(wd=odd), dict(wsc=None), dict(fmt=1), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(outs=-1),
                dict(act=2), dict(out=None), dict(dtype=3), dict(stride=7), dict(bias=ctypes.c_void_p((1 << 20) + 2))):
        assert prod(**bad) == INVALID, bad
    assert prod(rows=0) == 0 and prod(outs=0, stride=0) == 0
    assert lib.sr_microscale_values(None, P, 3, 4, 32, P, None) == INVALID and lib.sr_microscale_values(P, P, 0, 4, 32, P, None) == INVALID


def test_norm_refuses():
    lib = ops._library()
    odd = ctypes.c_void_p((1 << 20) + 1)

    def norm(x=P, res=None, w=None, eps=1e-6, dtype=1, rows=4, cols=64, xs=64, rs=64, total=None, out=P, fmt=1, scales=None):
        return lib.sr_rms_norm(x, res, w, eps, dtype, rows, cols, xs, rs, total, out, fmt, scales, None)
    for bad in (dict(x=None), dict(out=None), dict(dtype=3), dict(fmt=0), dict(rows=-1), dict(cols=0), dict(xs=-1), dict(res=P, rs=-1), dict(eps=-1.0),
                dict(eps=float("nan")), dict(fmt=3), dict(fmt=1, scales=P), dict(x=odd), dict(res=odd), dict(total=odd), dict(w=odd), dict(out=odd),
                dict(fmt=2, scales=ctypes.c_void_p((1 << 20) + 8)), dict(total=P, xs=65), dict(x=ctypes.c_void_p(1 << 21), res=P, total=P, rs=65)):
        assert norm(**bad) == INVALID, bad
    assert norm(rows=0, x=None) == 0


@pytest.mark.parametrize("rows, cols, fmt", [(1, 1, "mx4"), (129, 33, "mx4"), (128, 128, "mx8"), (300, 1000, "mx8"), (0, 5, "mx4")])
def test_sizes_are_those_of_the_layout(rows, cols, fmt):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert ops._library().sr_microscale_bytes(rows, cols, ops.FORMATS[fmt], ctypes.byref(a), ctypes.byref(b)) == 0
    m = sr.Microscaled.empty(rows, cols, fmt, "cpu")
    assert (m.data.numel(), m.scales.numel()) == (a.value, b.value)
    if rows:
        data, scales = oracle.pack(*oracle.quantize(np.ones((rows, cols)), fmt)[:2], fmt)
        assert (data.size, scales.size) == (a.value, b.value)
    assert sr.Microscaled(m.data, m.scales, rows, cols, fmt).rows == rows


def test_python_refuses_before_it_calls():
    x, w = torch.zeros(4, 64), torch.zeros(64)
    m = sr.Microscaled.empty(4, 64, "mx4", "cpu")
    for call in (lambda: sr.quantize(x), lambda: sr.rms_norm(x, w), lambda: sr.product(m, m), lambda: m.values(),
                 lambda: sr.linear_attention_step(torch.zeros(1, 2, 8), torch.zeros(1, 2, 8), torch.zeros(1, 2, 8), torch.zeros(2), torch.zeros(1, 2, 8, 8)),
                 lambda: sr.linear_attention_run(*[torch.zeros(3, 1, 2, 8)] * 3, torch.zeros(2))):
        with pytest.raises(SrError, match="CUDA device"):
            call()
    with pytest.raises(SrError, match="format"):
        sr.Microscaled(m.data, m.scales, 4, 64, "mx2")
    with pytest.raises(SrError, match="sizes"):
        sr.Microscaled(m.data, m.scales, 4, 96, "mx4")
    with pytest.raises(SrError, match="sizes"):
        sr.Microscaled(m.data[:, ::2], m.scales, 4, 64, "mx4")
    with pytest.raises(SrError, match="same format"):
        sr.product(m, sr.Microscaled.empty(4, 64, "mx8", "cpu"))


def test_oracle_rounds_to_nearest_even_and_never_saturates():
    v = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] + [0.0] * 24])
    code, scale, values = oracle.quantize(v, "mx4")
    assert scale[0, 0] == 127 and list(code[0, :8]) == [0, 2, 2, 4, 4, 6, 6, 7]
    for fmt, top in (("mx4", 6.0), ("mx8", 448.0)):
        for e in (-126, -40, 0, 60, 119 if fmt == "mx8" else 125):
            for f in (1.0, 1.0 + 2.0 ** -20):
                x = np.zeros((1, 32))
                x[0, 3] = top * f * 2.0 ** e
                _, scale, values = oracle.quantize(x, fmt)
                assert scale[0, 0] == e + 127 + (f > 1)
                assert abs(values[0, 3] - x[0, 3]) <= x[0, 3] * (0.25 if fmt == "mx4" else 2.0 ** -4)
