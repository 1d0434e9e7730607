"""The selective head's operators on layouts that allow units of 4, 8 and 16 bytes, with many sequences, against their definitions in 64 bits; the head in bf16; modes and slow paths of its calls."""
import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import SrError, selective
from tests import selective_bounds, selective_oracle as oracle
from tests.test_gpu_selective import DEV, DT, check_conv, head_oracle, head_weights, host, randn, spans, within

pytestmark = pytest.mark.gpu


def units(t, elements):
    """Whether rows of t (all but the last dimension) start on whole units of `elements`."""
    return t.data_ptr() % (elements * t.element_size()) == 0 and all(s % elements == 0 for s, n in zip(t.stride()[:-1], t.shape[:-1]) if n > 1)


def scan_inputs(lead, channels, states, groups, dtype, seed=0, softplus=True):
    """Rows of b and c start on 16 bytes where the states allow it, those of u, dt and z where the channels do."""
    low = randn(seed + 1, *lead, 8 + 2 * groups * states, dtype=dtype)
    b, c = (low[..., 8 + k * groups * states:8 + (k + 1) * groups * states].unflatten(-1, (groups, states)) for k in (0, 1))
    both = randn(seed + 2, *lead, 2 * channels, dtype=dtype)
    a = -torch.arange(1, states + 1, device=DEV).float() * torch.exp(0.2 * randn(seed + 3, channels, states))
    dt = randn(seed + 4, *lead, channels, dtype=dtype)
    return dict(u=both[..., :channels], dt=dt if softplus else (0.05 * dt.abs()).contiguous(), a=a.contiguous(), b=b, c=c), \
        dict(d=randn(seed + 5, channels), z=both[..., channels:], dt_bias=randn(seed + 6, channels) - 3.0 if softplus else None)


def check_scan(x, o, softplus, state, out, last, dtype, what=""):
    """x and o with frames and sequences."""
    want, e, left, es = selective_bounds.scan(*(host(x[k]) for k in ("u", "dt", "a", "b", "c")), **{k: None if v is None else host(v) for k, v in o.items()}, plus=softplus,
                                              state=None if state is None else host(state))
    within(host(out), want, e + oracle.HALF_STEP[dtype] * (np.abs(want) + e), (what, "out"))
    within(host(last), left, es, (what, "states"))


# ------------------------------------------------------------------------------------------ scan
RUNS = [  # frames, batch, channels, states, groups
    (1, 2, 40, 16, 1), (40, 2, 32, 8, 1), (37, 3, 48, 16, 2), (40, 2, 64, 24, 1), (33, 3, 40, 32, 1), (39, 2, 48, 64, 2), (40, 2, 40, 128, 1), (38, 5, 17, 16, 1), (40, 1, 64, 12, 1),
    (40, 2, 24, 4, 3), (333, 1, 16, 8, 1), (333, 2, 16, 16, 2), (333, 1, 16, 24, 1), (333, 1, 24, 32, 1), (333, 1, 33, 64, 1), (333, 1, 16, 128, 1), (600, 1, 20, 16, 1), (1100, 1, 8, 4, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sizes", RUNS, ids=str)
def test_scan_run_in_units(sizes, dtype):
    frames, batch, channels, states, groups = sizes
    vec = 16 // DT[dtype].itemsize
    assert (selective.scan_plan(DT[dtype], batch, frames, channels, states, groups)["segment"] > 0) == (frames > 300)
    state = randn(9, batch, channels, states)
    for softplus, gated, entering in ((True, True, state), (False, True, state), (False, False, None)):
        x, o = scan_inputs((frames, batch), channels, states, groups, dtype, softplus=softplus)
        assert states % vec or (units(x["b"], vec) and units(x["c"], vec))
        assert channels % vec or units(x["u"], vec)
        o["z"] = o["z"] if gated else None
        out, last = sr.selective_scan_run(**x, **o, softplus=softplus, state=entering)
        check_scan(x, o, softplus, entering, out, last, dtype, (softplus, gated))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("channels,states,groups", [(64, 16, 1), (48, 24, 2), (32, 64, 2), (24, 128, 1), (33, 32, 1)])
@pytest.mark.parametrize("lengths", [[0, 3, 900, 1, 40, 0], [7, 33, 0, 60]], ids=["one_long", "short"])
def test_scan_packed_in_units(lengths, channels, states, groups, dtype):
    at, offsets = spans(lengths)
    total = int(at[-1]) + 3
    x, o = scan_inputs((total,), channels, states, groups, dtype)
    state = randn(9, len(lengths), channels, states)
    kept = state.clone()
    out = torch.full((total, channels), 7.0, dtype=DT[dtype], device=DEV)
    sr.selective_scan_run(**x, **o, state=state, offsets=offsets, out=out, state_out=state)
    for b, n in enumerate(lengths):
        s = slice(at[b], at[b + 1])
        if n:
            check_scan({k: v if k == "a" else v[s][:, None] for k, v in x.items()}, dict(o, z=o["z"][s][:, None]), True, kept[b:b + 1], out[s][:, None], state[b:b + 1], dtype, b)
        else:
            assert torch.equal(state[b], kept[b])
    assert (out[int(at[-1]):] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("states,groups", [(4, 1), (8, 1), (16, 1), (16, 2), (20, 2), (64, 1), (128, 1), (5, 1), (70, 1)])
@pytest.mark.parametrize("batch", [1, 15, 16, 48, 70, 256])
def test_scan_steps_in_units_of_many_sequences(batch, states, groups, dtype):
    """Blocks go over 1, 3, 4 and 16 sequences, of 70 the last over two, with the loads of two or three under way."""
    channels = 10
    x, o = scan_inputs((3, batch), channels, states, groups, dtype)
    assert states % 8 or (units(x["b"], 8) and units(x["c"], 8))
    state = randn(9, batch, channels, states)
    first = state.clone()
    outs = torch.stack([sr.selective_scan_step(*(x[k] if k == "a" else x[k][t] for k in ("u", "dt", "a", "b", "c")), state, d=o["d"], z=o["z"][t], dt_bias=o["dt_bias"])
                        for t in range(3)])
    check_scan(x, o, True, first, outs, state, dtype)


# ------------------------------------------------------------------------------------------ convolution
@pytest.mark.parametrize("dtype,batch,channels,unit", [("bf16", 1, 264, 2), ("bf16", 31, 130, 2), ("bf16", 33, 264, 2), ("bf16", 70, 6, 2), ("bf16", 31, 2568, 4), ("bf16", 70, 1160, 4),
                                                       ("bf16", 33, 2404, 4), ("fp32", 1, 130, 2), ("fp32", 33, 264, 2), ("fp32", 70, 130, 2), ("bf16", 70, 1161, 1), ("fp32", 35, 33, 1)])
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 6, 7, 8])
def test_conv_steps_in_units(dtype, batch, channels, unit, width):
    """unit: channels that a thread has, by the number of values (at most 512 for each of the SMs' blocks: pairs of bf16) and where the rows start."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    if dtype == "bf16" and unit > 1:
        assert (batch * channels <= sms * 512) == (unit == 2)
    x, w, bias = randn(1, 3, batch, channels, dtype=dtype), randn(2, channels, width), randn(3, channels)
    assert unit == 1 or (units(x[0], unit) and channels % unit == 0)
    for given, silu in ((bias, True), (None, False)):
        state = randn(4, batch, width - 1, channels, dtype=dtype)
        first = state.clone()
        out = torch.stack([sr.causal_conv_step(x[t], w, state, bias=given, silu=silu) for t in range(3)])
        for b in {0, 1, 3, 4, batch // 2, batch - 2, batch - 1} & set(range(batch)):
            check_conv(x[:, b], w, given, silu, first[b], out[:, b], state[b], b, dtype)
        run, last = sr.causal_conv_run(x, w, bias=given, silu=silu, state=first)
        assert torch.equal(state, last) and torch.equal(out, run)


@pytest.mark.parametrize("dtype,channels", [("bf16", 136), ("fp32", 36), ("bf16", 1032)])
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 6, 7, 8])
def test_conv_packed_in_units(dtype, channels, width):
    lengths = [0, 1, 70, 2, 0, 133, 5, 0]
    at, offsets = spans(lengths)
    total = int(at[-1]) + 4
    x = randn(1, total, 2 * channels, dtype=dtype)[:, channels:]
    w, bias = randn(2, channels, width), randn(3, channels)
    state = randn(4, len(lengths), width - 1, channels, dtype=dtype)
    assert units(x, 16 // DT[dtype].itemsize)
    out = torch.full((total, channels), 7.0, dtype=DT[dtype], device=DEV)
    _, last = sr.causal_conv_run(x, w, bias=bias, silu=True, state=state, offsets=offsets, out=out)
    for b, n in enumerate(lengths):
        if n:
            check_conv(x[at[b]:at[b + 1]], w, bias, True, state[b], out[at[b]:at[b + 1]], last[b], b, dtype)
        else:
            assert torch.equal(last[b], state[b])
    assert (out[int(at[-1]):] == 7.0).all()


# ------------------------------------------------------------------------------------------ the head in bf16
@pytest.mark.parametrize("blocks,groups", [(1, 1), (2, 2)])
def test_head_in_bf16(blocks, groups):
    """A product's operand that another rounding to bf16 (2^-9 of it) puts on the other side of a border of its format (steps of up to 2^-3) is off by a step: one of 16 to 64, 2 % of the operands
    in the mean square, and of the product.  Five products follow each other in a block, two of them (convolution and gate, readout and norm) join two such errors, and one comes last:
    sqrt(5 + 2 + 1) * 2 % = 6 % of the outputs for a block, 8 % for two; twice that is allowed."""
    C, inner, N, rank, W, T, B, outs = 64, 96, 16, 4, 4, 40, 3, 10
    w = head_weights(C, inner, N, rank, W, groups, outs, blocks)
    head = sr.SelectiveHead(w, C, inner, N, rank, W, B, groups=groups, scale=0.5, format="mx8")
    assert head.tdtype is torch.bfloat16 and all(conv.dtype is torch.bfloat16 and scan.dtype is torch.float32 for conv, scan in head.get_state())
    x = randn(1, T, B, C, dtype="bf16").float()
    run = head.run(x)
    assert run.dtype is torch.float32 and run.shape == (T, B, outs)
    want = head_oracle(w, host(x), inner, N, rank, groups, "mx8", 0.5, 1e-6)
    allowed = (0.12 if blocks == 1 else 0.16) * np.sqrt((want ** 2).mean())
    assert np.sqrt(((host(run) - want) ** 2).mean()) <= allowed
    head.reset()
    assert torch.equal(head.run(x.bfloat16()), run)               # features of the head's own type
    head.reset()
    steps = torch.stack([head.step(x[t]) for t in range(T)])
    assert float((steps - run).square().mean().sqrt()) <= allowed
    head.reset()
    first, state = head.run(x[:17]), head.get_state()
    rest = head.run(x[17:])
    head.set_state(state)
    assert torch.equal(head.run(x[17:]), rest) and float((torch.cat((first, rest)) - run).square().mean().sqrt()) <= allowed


# ------------------------------------------------------------------------------------------ modes, and calls that the compiled module does not take
def calls(x):
    """Every call with x ([3][2][8]) among its inputs."""
    w, a, bc = torch.ones(8, 4, device=DEV), -torch.ones(8, 4, device=DEV), torch.ones(3, 2, 1, 4, device=DEV)
    y = torch.ones(3, 2, 8, device=DEV)
    taps, state = torch.ones(2, 3, 8, device=DEV), torch.ones(2, 8, 4, device=DEV)
    return [lambda: sr.causal_conv_run(x, w)[0], lambda: sr.causal_conv_step(x[0], w, taps), lambda: sr.causal_conv_run(y, w, bias=x[0, 0])[0],
            lambda: sr.selective_scan_run(x, y, a, bc, bc)[0], lambda: sr.selective_scan_run(y, x, a, bc, bc, z=x)[0], lambda: sr.selective_scan_run(y, y, a, bc, bc, d=x[0, 0])[0],
            lambda: sr.selective_scan_step(x[0], y[0], a, bc[0], bc[0], state), lambda: sr.selective_scan_step(y[0], y[0], a, bc[0], bc[0], state, z=x[0]),
            lambda: sr.block_norm(x[0], y[0])[0], lambda: sr.block_norm(y[0], x[0], gate=y[0])[0], lambda: sr.block_norm(y[0], y[0], gate=x[0])[0], lambda: sr.block_norm(y[0], y[0], x[0, 0])[0]]


def test_derivatives_are_refused_and_other_modes_taken():
    import torch.autograd.forward_ad as forward_ad
    x = randn(1, 3, 2, 8)
    want = [call() for call in calls(x)]
    for call in calls(x.clone().requires_grad_()):
        with pytest.raises(SrError, match="no backward pass"):
            call()
    with forward_ad.dual_level():
        for call in calls(forward_ad.make_dual(x, torch.ones_like(x))):
            with pytest.raises(SrError, match="no forward derivative"):
                call()
    for k in range(len(want)):
        with pytest.raises(SrError):
            torch.func.vmap(lambda y: calls(y)[k]())(x.expand(5, 3, 2, 8).contiguous())
        with pytest.raises(SrError):
            torch.func.jvp(lambda y: calls(y)[k](), (x,), (x,))
    with torch.no_grad():
        assert all(torch.equal(call(), one) for call, one in zip(calls(x.clone().requires_grad_()), want))
    with torch.inference_mode():
        assert all(torch.equal(call(), one) for call, one in zip(calls(x.clone()), want))


FAST = ("conv_run", "conv_step", "scan_run", "scan_step", "block_norm")


def test_calls_without_the_compiled_module_are_the_same(monkeypatch):
    """As on a device that is not the current one."""
    lengths = [3, 0, 400, 5]
    at, offsets = spans(lengths)
    T, B, C, N, G = int(at[-1]), len(lengths), 24, 16, 2
    results = []
    for compiled in (True, False):
        if not compiled:
            for name in FAST:
                monkeypatch.setattr(selective._compiled, name, lambda *_: None)
        got = []
        for dtype in ("bf16", "fp32"):
            x, o = scan_inputs((T,), C, N, G, dtype)
            y, p = scan_inputs((60, B), C, N, G, dtype, seed=20)
            state, taps, w, bias = randn(9, B, C, N), randn(10, B, 3, C, dtype=dtype), randn(11, C, 4), randn(12, C)
            kept, conv = torch.full((T, C), 7.0, dtype=DT[dtype], device=DEV), torch.full((T, C), 7.0, dtype=DT[dtype], device=DEV)
            got += sr.selective_scan_run(**x, **o, state=state, offsets=offsets) + sr.selective_scan_run(**y, **p) + sr.selective_scan_run(**y, softplus=False, d=p["d"])         # (the last one grows beyond all bounds)
            got += sr.causal_conv_run(x["u"], w, bias=bias, silu=True, state=taps, offsets=offsets) + sr.causal_conv_run(y["u"], w)
            got.append(sr.selective_scan_step(*(v if k == "a" else v[0] for k, v in y.items()), state, d=p["d"], z=p["z"][0], dt_bias=p["dt_bias"]))
            got.append(sr.causal_conv_step(y["u"][0], w, taps, bias=bias, silu=True))
            got += [state.clone(), taps.clone()]
            versions = [t._version for t in (state, taps, kept, conv)]
            sr.selective_scan_run(**x, **o, state=state, offsets=offsets, out=kept, state_out=state)
            sr.causal_conv_run(x["u"], w, state=taps, offsets=offsets, out=conv, state_out=taps)
            assert [t._version for t in (state, taps, kept, conv)] == [v + 1 for v in versions]
            got += [kept, conv, state, taps]
            r = randn(13, 50, 96, dtype=dtype)
            for norms in ("both", "after", "before", "none"):
                h = sr.block_norm(r, r.flip(0), torch.ones(96, device=DEV), None, gate=r, gate_act="silu", scale=0.3, norms=norms)
                got += h if isinstance(h, tuple) else (h,)
            for format in ("mx4", "mx8"):
                m, h = sr.block_norm(r[:, :70], r[:, 3:73], gate=None, format=format)
                got += [m.data, m.values(), h]                # (scales are padded to whole tiles with anything)
        results.append(got)
    assert len(results[0]) == len(results[1])
    for k, (a, b) in enumerate(zip(*results)):
        torch.testing.assert_close(a, b, rtol=0, atol=0, equal_nan=True, msg=str(k))


@pytest.mark.parametrize("kind", ["selective", "temporal"])
def test_heads_made_in_inference_mode_run_outside_of_it(kind):
    from tests.test_operator_refusals import weights
    with torch.inference_mode():
        head = sr.SelectiveHead(head_weights(32, 32, 8, 2, 4, 1, 3, 1), 32, 32, 8, 2, 4, 2) if kind == "selective" else sr.TemporalHead(weights(channels=32), 32, 4, 2, 32, 48, 2)
        x = randn(2, 5, 2, 32)
        one = head.run(x)
        head.reset()
    assert torch.equal(head.run(x), one)
    state = head.get_state()
    head.reset()
    assert torch.equal(head.run(x), one)
    head.set_state(state)
    with torch.inference_mode():
        head.reset()
        assert torch.equal(head.run(x), one)
