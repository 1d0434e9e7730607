"""Refusals, sizes and argument checks of the selective head's operators: nothing here reaches a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import SrError, operators as ops, selective
from tests import selective_oracle as oracle

INVALID, UNSUPPORTED = 1, 5
P = ctypes.c_void_p(1 << 20)                      # never read: every call here is refused, or has nothing to do
P2 = ctypes.c_void_p(1 << 21)
ODD = ctypes.c_void_p((1 << 20) + 1)


def conv_desc(dtype=1, batch=2, channels=64, width=4, act=1, frames=8, **strides):
    d = selective._ConvDesc(dtype, batch, channels, width, act, frames)
    for name in ("x", "out"):
        setattr(d, name, selective._FrameStrides(*strides.get(name, (batch * channels, channels))))
    return d


def conv_run(d, x=P, weight=P, bias=None, offsets=None, s_in=None, s_out=None, out=P2):
    return selective._library().sr_causal_conv_run(ctypes.byref(d) if d else None, x, weight, bias, offsets, s_in, s_out, out, None)


def conv_step(d, x=P, weight=P, bias=None, state=P, out=P2):
    return selective._library().sr_causal_conv_step(ctypes.byref(d) if d else None, x, weight, bias, state, out, None)


@pytest.mark.parametrize("call", [conv_run, conv_step])
def test_conv_refuses_sizes_and_pointers(call):
    assert call(None) == INVALID
    for bad in (dict(dtype=2), dict(batch=-1), dict(channels=0), dict(width=0), dict(act=2), dict(frames=-1), dict(x=(-1, 1)), dict(out=(1, -1))):
        assert call(conv_desc(**bad)) == INVALID, bad
    assert call(conv_desc(width=9)) == UNSUPPORTED
    for name in ("x", "weight", "out"):
        assert call(conv_desc(), **{name: None}) == INVALID, name
    for name in ("x", "weight", "out", "bias"):
        assert call(conv_desc(), **{name: ODD}) == INVALID, name
    assert call(conv_desc(), out=P) == INVALID
    assert call(conv_desc(batch=0)) == 0
    assert conv_run(conv_desc(), s_in=ODD) == INVALID and conv_run(conv_desc(), s_out=ODD) == INVALID and conv_run(conv_desc(), offsets=ODD) == INVALID
    assert conv_step(conv_desc(), state=None) == INVALID and conv_step(conv_desc(), state=ODD) == INVALID
    assert conv_run(conv_desc(frames=0), x=None, out=None) == 0


def scan_desc(dtype=1, batch=2, channels=64, states=16, groups=2, softplus=1, frames=8, **strides):
    d = selective._ScanDesc(dtype, batch, channels, states, groups, softplus, frames)
    for name in ("u", "dt", "z", "out"):
        setattr(d, name, selective._FrameStrides(*strides.get(name, (batch * channels, channels))))
    for name in ("b", "c"):
        setattr(d, name, ops._Strides(*strides.get(name, (batch * 64, 64, 16))))
    return d


def scan_run(d, u=P, dt=P, a=P, b=P, c=P, skip=None, z=None, bias=None, offsets=None, s_in=None, s_out=None, out=P2, ws=None, size=0):
    return selective._library().sr_selective_scan_run(ctypes.byref(d) if d else None, u, dt, a, b, c, skip, z, bias, offsets, s_in, s_out, out, ws, size, None)


def scan_step(d, u=P, dt=P, a=P, b=P, c=P, skip=None, z=None, bias=None, state=P, out=P2):
    return selective._library().sr_selective_scan_step(ctypes.byref(d) if d else None, u, dt, a, b, c, skip, z, bias, state, out, None)


@pytest.mark.parametrize("call", [scan_run, scan_step])
def test_scan_refuses_sizes_and_pointers(call):
    assert call(None) == INVALID
    for bad in (dict(dtype=2), dict(batch=-1), dict(channels=0), dict(states=0), dict(groups=0), dict(groups=3), dict(softplus=2), dict(frames=-1), dict(u=(-1, 1)),
                dict(dt=(1, -1)), dict(z=(-1, 0)), dict(out=(1, -1)), dict(b=(0, 0, -1)), dict(c=(-1, 0, 0))):
        assert call(scan_desc(**bad)) == INVALID, bad
    assert call(scan_desc(states=129)) == UNSUPPORTED
    for name in ("u", "dt", "a", "b", "c", "out"):
        assert call(scan_desc(), **{name: None}) == INVALID, name
    for name in ("u", "dt", "a", "b", "c", "out", "skip", "z", "bias"):
        assert call(scan_desc(), **{name: ODD}) == INVALID, name
    for name in ("u", "dt", "b", "c", "z"):
        assert call(scan_desc(), **{name: P2}) == INVALID, name      # the outputs would lie on them
    assert call(scan_desc(batch=0)) == 0
    two = ctypes.c_void_p((1 << 20) + 2)
    assert scan_run(scan_desc(), s_in=two) == INVALID and scan_run(scan_desc(), s_out=two) == INVALID and scan_run(scan_desc(), offsets=two) == INVALID
    assert scan_step(scan_desc(), state=None) == INVALID and scan_step(scan_desc(), state=two) == INVALID
    assert scan_run(scan_desc(frames=0), u=None, out=None) == 0
    size = ctypes.c_size_t()
    assert selective._library().sr_selective_scan_workspace_bytes(ctypes.byref(scan_desc()), 0, None) == INVALID
    assert selective._library().sr_selective_scan_workspace_bytes(ctypes.byref(scan_desc(states=200)), 0, ctypes.byref(size)) == UNSUPPORTED


def block_desc(dtype=1, norms=3, act=1, format=1, scale=1.0, eps=1e-6, rows=4, cols=64, ys=64, rs=64, gs=64):
    return selective._BlockDesc(dtype, norms, act, format, scale, eps, rows, cols, ys, rs, gs)


def block(d, y=P, r=P, gate=None, after=None, before=None, h=P2, out=ctypes.c_void_p(1 << 22), scales=None):
    return selective._library().sr_block_norm(ctypes.byref(d) if d else None, y, r, gate, after, before, h, out, scales, None)


def test_block_norm_refuses():
    assert block(None) == INVALID
    for bad in (dict(dtype=2), dict(norms=4), dict(norms=-1), dict(act=3), dict(act=-1), dict(format=0), dict(format=4), dict(eps=-1.0), dict(eps=float("nan")), dict(rows=-1),
                dict(cols=0), dict(rows=1 << 31), dict(cols=1 << 31), dict(ys=-1), dict(rs=-1)):
        assert block(block_desc(**bad)) == INVALID, bad
    assert block(block_desc(gs=-1), gate=P) == INVALID
    for name in ("y", "r", "h", "out"):
        assert block(block_desc(), **{name: None}) == INVALID, name
    for name in ("y", "r", "h", "out", "gate", "after", "before"):
        assert block(block_desc(), **{name: ODD}) == INVALID, name
    assert block(block_desc(), h=P) == INVALID and block(block_desc(), out=P) == INVALID and block(block_desc(), out=P2) == INVALID
    assert block(block_desc(norms=1)) == INVALID                     # an output without its norm
    assert block(block_desc(), scales=P) == INVALID and block(block_desc(format=2)) == INVALID and block(block_desc(format=2), scales=ODD) == INVALID
    assert block(block_desc(rows=0)) == 0


def test_python_refuses_what_is_not_on_a_gpu_or_wants_a_gradient():
    x, w = torch.zeros(4, 2, 8), torch.zeros(8, 4)
    a, bc = torch.zeros(8, 16), torch.zeros(4, 2, 1, 16)
    calls = [lambda x: sr.causal_conv_run(x, w), lambda x: sr.causal_conv_step(x[0], w, torch.zeros(2, 3, 8)), lambda x: sr.selective_scan_run(x, x, a, bc, bc),
             lambda x: sr.selective_scan_step(x[0], x[0], a, bc[0], bc[0], torch.zeros(2, 8, 16)), lambda x: sr.block_norm(x[0], x[0])]
    for call in calls:
        with pytest.raises(SrError, match="CUDA"):
            call(x)
        with pytest.raises(SrError, match="backward"):
            call(x.clone().requires_grad_())
        with pytest.raises(SrError, match="tensors are required"):
            call([None])
        with torch.autograd.forward_ad.dual_level(), pytest.raises(SrError, match="derivative"):
            call(torch.autograd.forward_ad.make_dual(x, x))


def test_scan_plans_need_no_device():
    for states in (1, 4, 5, 16, 100, 128):
        p = selective.scan_plan(torch.bfloat16, 4, 1000, 512, states, sms=148)
        assert p["held"] * p["lanes"] >= states and p["segment"] >= 0
    with pytest.raises(SrError):
        selective.scan_plan(torch.bfloat16, 4, 1000, 512, 129, sms=148)


def test_scan_plans_cut_what_leaves_schedulers_idle():
    def plan(batch, frames, channels, states=16, packed=False, dtype=torch.bfloat16):
        return selective.scan_plan(dtype, batch, frames, channels, states, packed=packed, sms=148)

    assert plan(32, 128, 2048)["segment"] == 0                    # enough channels
    assert plan(1, 32, 64)["segment"] == 0                        # too short
    for batch, frames, channels in ((1, 16384, 1024), (5, 500, 1111), (1, 300, 8)):
        p = plan(batch, frames, channels)
        assert p["segment"] % 8 == 0 and p["segments"] == batch * -(-frames // p["segment"]) and p["segment"] < frames
    p = plan(16, 16384, 1024, packed=True)
    assert p["segment"] % 8 == 0 and p["segments"] == 16384 // p["segment"] + 16
    assert {(plan(1, 64, 64, n)["held"], plan(1, 64, 64, n)["lanes"]) for n in (4, 8, 12, 16, 24, 32, 64, 128)} == {(4, 1), (8, 1), (12, 1), (16, 1), (12, 2), (16, 2), (16, 4), (16, 8)}
    for big in (dict(frames=1 << 50, channels=64), dict(frames=8, channels=1 << 30, batch=1 << 30)):
        with pytest.raises(SrError):
            plan(**dict(dict(batch=1), **big))


def test_oracle_scan_is_the_sum_it_stands_for():
    rng = np.random.default_rng(0)
    T, C, N = 7, 4, 3
    u, dt, a, b, c = rng.standard_normal((T, C)), rng.standard_normal((T, C)), -rng.random((C, N)), rng.standard_normal((T, 2, N)), rng.standard_normal((T, 2, N))
    out, h, mag, m, top = oracle.scan(u, dt, a, b, c)
    r = np.log(1 + np.exp(dt))
    for t in range(T):
        for i in range(C):
            want = sum(c[t, i // 2, n] * np.exp(a[i, n] * r[s + 1:t + 1, i].sum()) * r[s, i] * u[s, i] * b[s, i // 2, n] for s in range(t + 1) for n in range(N))
            assert abs(want - out[t, i]) < 1e-12
    x, w = rng.standard_normal((T, C)), rng.standard_normal((C, 3))
    y, last, _ = oracle.conv(x, w)
    assert np.allclose(y[5], sum(w[:, j] * x[3 + j] for j in range(3))) and np.array_equal(last, x[-2:]) and np.allclose(y[0], w[:, 2] * x[0])


def test_head_refuses_sizes():
    for bad in (dict(states=129), dict(width=9), dict(inner=7, groups=2), dict(rank=0), dict(batch=-1), dict(format="x"), dict(dtype="fp16"), dict(eps=-1.0)):
        args = dict(channels=8, inner=8, states=4, rank=1, width=4, batch=1, device="cpu")
        args.update(bad)
        with pytest.raises(SrError):
            sr.SelectiveHead({"blocks": [{}]}, **args)
    with pytest.raises(SrError, match="blocks"):
        sr.SelectiveHead({}, 8, 8, 4, 1, 4, 1, device="cpu")
    with pytest.raises(SrError, match="missing"):
        sr.SelectiveHead({"blocks": [{}]}, 8, 8, 4, 1, 4, 1, device="cpu")
