"""The selective head's operators against their definitions in 64 bits, and the head itself, on the GPU."""
import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import selective
from tests import operator_oracle, selective_oracle as oracle

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
DEV = "cuda:0"


def host(t):
    return t.detach().double().cpu().numpy()


def randn(seed, *shape, dtype="fp32"):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).to(DEV)


def within(got, want, bound, what=""):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - want) / np.maximum(bound, 1e-300))), np.argwhere(bad)[:3].tolist())


def spans(lengths):
    at = np.concatenate(([0], np.cumsum(lengths)))
    return at, torch.tensor(at, dtype=torch.int64, device=DEV)


# ------------------------------------------------------------------------------------------ convolution
def check_conv(x, w, bias, silu, state, out, last, b, dtype):
    """One sequence."""
    want, left, mag = oracle.conv(host(x), host(w), None if bias is None else host(bias), silu, None if state is None else host(state))
    # W products and sums, the activation's own error, and its slope of at most 1.1
    within(host(out), want, oracle.HALF_STEP[dtype] * np.abs(want) + 1.2 * (w.shape[1] + 2) * 2.0 ** -24 * mag + (2.0 ** -21 if dtype == "fp32" else 2.0 ** -18) * np.abs(want) + 1e-37, b)
    assert np.array_equal(host(last), left), b


@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("dtype,channels", [("bf16", 136), ("bf16", 65), ("fp32", 36), ("fp32", 129)])
def test_conv_run(width, dtype, channels):
    for frames, batch, given, silu in ((1, 3, True, True), (7, 2, False, True), (40, 3, True, False), (131, 1, True, True)):
        x, w = randn(1, frames, batch, channels, dtype=dtype), randn(2, channels, width)
        bias = randn(3, channels) if given else None
        state = randn(4, batch, width - 1, channels, dtype=dtype) if given else None
        out, last = sr.causal_conv_run(x, w, bias=bias, silu=silu, state=state)
        for b in range(batch):
            check_conv(x[:, b], w, bias, silu, None if state is None else state[b], out[:, b], last[b], b, dtype)


@pytest.mark.parametrize("dtype,channels,width", [("bf16", 264, 4), ("fp32", 33, 3), ("bf16", 17, 8)])
def test_conv_packed_in_place_and_strided(dtype, channels, width):
    lengths = [0, 1, 70, 2, 0, 33, 5, 0]
    at, offsets = spans(lengths)
    total = int(at[-1]) + 4                                      # frames that no sequence has
    x = randn(1, total, 2 * channels + 8, dtype=dtype)[:, 8:8 + channels]
    w, bias = randn(2, channels, width), randn(3, channels)
    state = randn(4, len(lengths), width - 1, channels, dtype=dtype)
    kept = state.clone()
    out = torch.full((total, channels), 7.0, dtype=DT[dtype], device=DEV)
    got, last = sr.causal_conv_run(x, w, bias=bias, silu=True, state=state, offsets=offsets, out=out, state_out=state)
    assert got is out and last is state
    for b, n in enumerate(lengths):
        if n:
            check_conv(x[at[b]:at[b + 1]], w, bias, True, kept[b], out[at[b]:at[b + 1]], state[b], b, dtype)
        else:
            assert torch.equal(state[b], kept[b])
    assert (out[int(at[-1]):] == 7.0).all()


@pytest.mark.parametrize("dtype,channels,width,batch", [("bf16", 264, 4, 3), ("fp32", 33, 3, 5), ("bf16", 17, 8, 1), ("fp32", 8, 1, 2), ("bf16", 1032, 2, 70)])
def test_conv_steps_are_a_run(dtype, channels, width, batch):
    x, w, bias = randn(1, 6, batch, channels + 3, dtype=dtype)[..., :channels], randn(2, channels, width), randn(3, channels)
    state = randn(4, batch, width - 1, channels, dtype=dtype)
    out, last = sr.causal_conv_run(x, w, bias=bias, silu=True, state=state)
    steps = torch.stack([sr.causal_conv_step(x[t], w, state, bias=bias, silu=True) for t in range(6)])
    assert torch.equal(steps, out) and torch.equal(state, last)


# ------------------------------------------------------------------------------------------ scan
def scan_inputs(frames, batch, channels, states, groups, dtype, packed=False, seed=0):
    lead = (frames,) if packed else (frames, batch)
    low = randn(seed + 1, *lead, 5 + 2 * groups * states, dtype=dtype)
    b, c = (low[..., 5 + k * groups * states:5 + (k + 1) * groups * states].unflatten(-1, (groups, states)) for k in (0, 1))
    both = randn(seed + 2, *lead, 2 * channels, dtype=dtype)
    a = -torch.arange(1, states + 1, device=DEV).float() * torch.exp(0.2 * randn(seed + 3, channels, states))
    return dict(u=both[..., :channels], dt=randn(seed + 4, *lead, channels, dtype=dtype), a=a.contiguous(), b=b, c=c), \
        dict(d=randn(seed + 5, channels), z=both[..., channels:], dt_bias=randn(seed + 6, channels) - 3.0)


def check_scan(x, o, softplus, state, out, last, what, dtype):
    """One sequence, x and o with its frames only."""
    opt = {k: None if v is None else host(v) for k, v in o.items()}
    want, left, mag, m, top = oracle.scan(*(host(x[k]) for k in ("u", "dt", "a", "b", "c")), **opt, plus=softplus, state=None if state is None else host(state))
    e = oracle.scan_error(want.shape[0], x["a"].shape[1], top)
    within(host(out), want, oracle.HALF_STEP[dtype] * np.abs(want) + e * mag + 1e-30, what)
    within(host(last), left, e * m + 1e-30, what)


SCANS = [  # frames, batch, channels, states, groups
    (1, 2, 40, 16, 1), (2, 1, 128, 16, 1), (9, 3, 65, 16, 5), (64, 2, 300, 16, 1), (130, 1, 33, 16, 1), (37, 2, 64, 1, 1), (37, 2, 64, 3, 2), (50, 2, 70, 4, 1), (50, 2, 70, 5, 2),
    (70, 2, 129, 8, 1), (70, 2, 34, 12, 2), (70, 1, 34, 24, 2), (70, 2, 48, 32, 3), (40, 2, 48, 64, 2), (40, 1, 40, 100, 4), (33, 2, 18, 128, 1), (300, 1, 1, 16, 1), (600, 1, 20, 16, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sizes", SCANS, ids=str)
def test_scan_run(sizes, dtype):
    frames, batch, channels, states, groups = sizes
    x, o = scan_inputs(frames, batch, channels, states, groups, dtype)
    state = randn(9, batch, channels, states)
    for options, softplus, entering in ((o, True, state), (dict(d=None, z=None, dt_bias=None), True, None), (dict(o, z=None), True, state)):
        out, last = sr.selective_scan_run(**x, **options, softplus=softplus, state=entering)
        for i in range(batch):
            one = {k: v if k == "a" else v[:, i] for k, v in x.items()}
            check_scan(one, dict(options, z=None if options["z"] is None else options["z"][:, i]), softplus, None if entering is None else entering[i], out[:, i], last[i], i, dtype)


def test_scan_without_softplus_and_with_growing_states():
    x, o = scan_inputs(20, 2, 24, 16, 1, "fp32")
    x["dt"] = x["dt"] * 0.1                                       # steps of both signs: some states grow
    out, last = sr.selective_scan_run(**x, d=o["d"], z=None, dt_bias=None, softplus=False)
    for i in range(2):
        check_scan({k: v if k == "a" else v[:, i] for k, v in x.items()}, dict(d=o["d"], z=None, dt_bias=None), False, None, out[:, i], last[i], i, "fp32")


@pytest.mark.parametrize("dtype,channels,states,groups", [("bf16", 72, 16, 1), ("fp32", 33, 12, 3), ("bf16", 16, 64, 2)])
def test_scan_packed_in_place(dtype, channels, states, groups):
    lengths = [0, 1, 170, 2, 0, 33, 700, 0]
    at, offsets = spans(lengths)
    total = int(at[-1]) + 3
    x, o = scan_inputs(total, len(lengths), channels, states, groups, dtype, packed=True)
    state = randn(9, len(lengths), channels, states)
    kept = state.clone()
    out = torch.full((total, channels), 7.0, dtype=DT[dtype], device=DEV)
    got, last = sr.selective_scan_run(**x, **o, state=state, offsets=offsets, out=out, state_out=state)
    assert got is out and last is state
    for b, n in enumerate(lengths):
        s = slice(at[b], at[b + 1])
        if n:
            check_scan({k: v if k == "a" else v[s] for k, v in x.items()}, dict(o, z=o["z"][s]), True, kept[b], out[s], state[b], b, dtype)
        else:
            assert torch.equal(state[b], kept[b])
    assert (out[int(at[-1]):] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("batch,channels,states,groups", [(1, 40, 16, 1), (3, 65, 5, 5), (17, 72, 16, 2), (40, 33, 4, 1), (2, 20, 128, 2), (18, 6, 100, 3), (5, 300, 1, 1), (2, 10, 70, 1)])
def test_scan_steps(batch, channels, states, groups, dtype):
    x, o = scan_inputs(3, batch, channels, states, groups, dtype)
    state = randn(9, batch, channels, states)
    first = state.clone()
    outs = torch.stack([sr.selective_scan_step(*(x[k] if k == "a" else x[k][t] for k in ("u", "dt", "a", "b", "c")), state, d=o["d"], z=o["z"][t], dt_bias=o["dt_bias"])
                        for t in range(3)])
    for i in range(batch):
        one = {k: v if k == "a" else v[:, i] for k, v in x.items()}
        check_scan(one, dict(o, z=o["z"][:, i]), True, first[i], outs[:, i], state[i], i, dtype)


def test_scan_runs_twice_alike_and_goes_on():
    x, o = scan_inputs(100, 2, 48, 16, 1, "fp32")
    whole, last = sr.selective_scan_run(**x, **o)
    again, same = sr.selective_scan_run(**x, **o)
    assert torch.equal(whole, again) and torch.equal(last, same)
    cut = [{k: v if k == "a" else v[s] for k, v in x.items()} for s in (slice(0, 37), slice(37, 100))]
    o1, s1 = sr.selective_scan_run(**cut[0], **dict(o, z=o["z"][:37]))
    o2, s2 = sr.selective_scan_run(**cut[1], **dict(o, z=o["z"][37:]), state=s1)
    torch.testing.assert_close(torch.cat((o1, o2)), whole, rtol=1e-4, atol=1e-5)
    torch.testing.assert_close(s2, last, rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("what,value", [("u", float("inf")), ("u", float("nan")), ("dt", float("nan")), ("dt", float("inf")), ("z", float("nan")), ("dt", float("-inf"))])
def test_scan_what_is_not_finite_stays_in_its_channel(what, value):
    x, o = scan_inputs(90, 2, 40, 12, 2, "fp32")
    clean, last = sr.selective_scan_run(**x, **o)
    at = dict(x, **o)[what]
    at[30, 1, 7] = value
    out, left = sr.selective_scan_run(**x, **o)
    keep = torch.ones(2, 40, dtype=torch.bool, device=DEV)
    keep[1, 7] = False
    assert torch.equal(out[:, keep], clean[:, keep]) and torch.equal(left[keep], last[keep])
    assert torch.equal(out[:30], clean[:30])
    if what == "dt" and value < 0:                                # a step of nothing
        want, h, mag, m, top = oracle.scan(*(host(x[k] if k == "a" else x[k][:, 1]) for k in ("u", "dt", "a", "b", "c")), host(o["d"]), host(o["z"][:, 1]), host(o["dt_bias"]))
        within(host(out[:, 1, 7]), want[:, 7], oracle.scan_error(90, 12, top) * mag[:, 7] + 1e-30)
    elif what == "z":
        assert torch.isnan(out[30, 1, 7]) and torch.equal(left, last)
    else:
        assert not torch.isfinite(out[30, 1, 7])


def longer(frames, states, groups, dtype, seed=0):
    """One sequence that is cut into segments."""
    x, o = scan_inputs(frames, 1, 2 * groups, states, groups, dtype, seed=seed)
    plan = selective.scan_plan(DT[dtype], 1, frames, 2 * groups, states, groups)
    assert 0 < plan["segment"] < frames and plan["held"] * plan["lanes"] >= states
    return x, o


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("states,groups", [(3, 1), (8, 2), (12, 1), (16, 3), (24, 1), (32, 1), (60, 1), (128, 1)])
def test_scan_in_segments_and_in_place(states, groups, dtype):
    x, o = longer(333, states, groups, dtype)
    state = randn(9, 1, 2 * groups, states)
    kept = state.clone()
    out, last = sr.selective_scan_run(**x, **o, state=state, state_out=state)
    assert last is state
    check_scan({k: v if k == "a" else v[:, 0] for k, v in x.items()}, dict(o, z=o["z"][:, 0]), True, kept[0], out[:, 0], state[0], (states, groups), dtype)


def test_scan_states_do_not_drift():
    """4000 frames of states that lose a ten-thousandth to a hundredth of themselves in each: a chunk's 32 approximate exponentials (2^-22 each) enter a value once, the rest are carried
    over by chunks, with 2^-23 and a rounding each."""
    T, C, N = 4000, 8, 16
    x, o = scan_inputs(T, 1, C, N, 1, "fp32")
    x["a"] = -(10.0 ** torch.linspace(-2, 0, N, device=DEV)).repeat(C, 1).contiguous()
    x["dt"] = 0.01 * (1 + 0.3 * torch.rand(T, 1, C, generator=torch.Generator().manual_seed(5)).to(DEV))
    x["u"] = x["u"].abs() + 0.5
    x["b"] = x["b"].abs() + 0.1                                   # (no cancellation: the sums are their terms' magnitudes)
    out, last = sr.selective_scan_run(**x, softplus=False)
    _, want, _, m, _ = oracle.scan(*(host(x[k] if k == "a" else x[k][:, 0]) for k in ("u", "dt", "a", "b", "c")), plus=False)
    # exponents add up to 0.4 to 50: an exponent's rounding is 2^-23 of it, of which a state that has lost e^-s keeps s e^-s < 1
    within(host(last[0]), want, (32 * 2.0 ** -22 + T / 32 * 2 * 2.0 ** -23 + 2.0 ** -21) * m)


@pytest.mark.parametrize("lengths", [[0, 3, 900, 1, 40, 0], [60] * 9 + [0, 64, 1], [0, 0, 0, 400, 0]], ids=["one_long", "none_long", "all_in_one"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scan_packed_cut_where_one_is_long(lengths, dtype):
    at, offsets = spans(lengths)
    total, C = int(at[-1]), 24
    x, o = scan_inputs(total, len(lengths), C, 16, 2, dtype, packed=True)
    assert selective.scan_plan(DT[dtype], len(lengths), total, C, 16, 2, packed=True)["segment"] > 0
    state = randn(9, len(lengths), C, 16)
    kept = state.clone()
    out, _ = sr.selective_scan_run(**x, **o, state=state, offsets=offsets, state_out=state)
    for b, n in enumerate(lengths):
        s = slice(at[b], at[b + 1])
        if n:
            check_scan({k: v if k == "a" else v[s] for k, v in x.items()}, dict(o, z=o["z"][s]), True, kept[b], out[s], state[b], b, dtype)
        else:
            assert torch.equal(state[b], kept[b])


@pytest.mark.parametrize("states", [16, 15])
def test_scan_packed_cut_with_many_states(states):
    lengths = [1, 0, 5] * 14 + [700, 2]
    at, offsets = spans(lengths)
    total, C = int(at[-1]), 1024
    x, o = scan_inputs(total, len(lengths), C, states, 1, "bf16", packed=True)
    assert 0 < selective.scan_plan(torch.bfloat16, len(lengths), total, C, states, packed=True)["segment"] < 300
    state = randn(9, len(lengths), C, states)
    out, last = sr.selective_scan_run(**x, **o, state=state, offsets=offsets)
    for b in (0, 1, 2, 41, 42, 43):
        s = slice(at[b], at[b + 1])
        if lengths[b]:
            check_scan({k: v if k == "a" else v[s] for k, v in x.items()}, dict(o, z=o["z"][s]), True, state[b], out[s], last[b], b, "bf16")
        else:
            assert torch.equal(last[b], state[b])


def test_scan_in_segments_of_thousands_of_frames():
    """The same inputs in every frame, so that frame t's state is x (1 - q^t) / (1 - q), q = exp(r a).  A state remembers 1000 frames at most: 32 approximate exponentials (2^-22 each), 1000 / 32
    carries (2^-23, and a rounding, each), the steps' sums (32 roundings of a chunk's, which is 1 over all that is remembered), and a few roundings of the output's sum."""
    lengths, C, N = [119000, 0, 1000], 2048, 4
    at, offsets = spans(lengths)
    T = int(at[-1])
    plan = selective.scan_plan(torch.bfloat16, len(lengths), T, C, N, packed=True)
    assert plan["segment"] > 1024
    a = -(10.0 ** torch.linspace(-1, 0, N, device=DEV)).repeat(C, 1).contiguous()
    u, dt, b, c = (randn(k, *s, dtype="bf16").abs() for k, s in enumerate(((C,), (C,), (1, N), (1, N))))
    dt = (0.01 + 0.03 * dt.float().clamp(max=1.0)).bfloat16()
    state = randn(9, len(lengths), C, N).abs()
    out, last = sr.selective_scan_run(u.expand(T, C), dt.expand(T, C), a, b.expand(T, 1, N), c.expand(T, 1, N), softplus=False, state=state, offsets=offsets)
    e = 32 * 2.0 ** -22 + (1000 / 32 + 1) * 2 * 2.0 ** -23 + 32 * 2.0 ** -23 + 2.0 ** -21
    some = slice(0, C, 37)
    for s, n in enumerate(lengths):
        times = np.unique(np.concatenate([np.arange(1, min(n, 3)), np.arange(1, n + 1, 311), plan["segment"] * np.arange(1, n // plan["segment"] + 1), [n]]))[:, None, None] if n else np.zeros((1, 1, 1))
        r, A, x = host(dt[some])[None, :, None], host(a[some])[None], host(dt[some])[None, :, None] * host(u[some])[None, :, None] * host(b)[None]
        grown = -np.expm1(r * A * times)                          # 1 - q^t
        h = (1 - grown) * host(state[s, some])[None] + x * grown / -np.expm1(r * A)
        if n:
            want = (h * host(c)[None]).sum(-1)
            within(host(out[at[s]:at[s + 1]][torch.from_numpy(times[:, 0, 0] - 1).to(DEV)][:, some]), want, oracle.HALF_STEP["bf16"] * want + e * want, s)
        within(host(last[s, some]), h[-1], e * h[-1], s)


def test_many_short_sequences():
    rng = np.random.default_rng(3)
    lengths = rng.integers(0, 6, 1500).tolist() + [300]
    at, offsets = spans(lengths)
    total, C = int(at[-1]), 10
    x, o = scan_inputs(total, len(lengths), C, 4, 1, "fp32", packed=True)
    state, taps = randn(9, len(lengths), C, 4), randn(10, len(lengths), 3, C)
    w = randn(11, C, 4)
    out, last = sr.selective_scan_run(**x, **o, state=state, offsets=offsets)
    conv, left = sr.causal_conv_run(x["u"], w, silu=True, state=taps, offsets=offsets)
    for b in list(range(0, 1500, 61)) + [1499, 1500]:
        s = slice(at[b], at[b + 1])
        if lengths[b]:
            check_scan({k: v if k == "a" else v[s] for k, v in x.items()}, dict(o, z=o["z"][s]), True, state[b], out[s], last[b], b, "fp32")
            check_conv(x["u"][s], w, None, True, taps[b], conv[s], left[b], b, "fp32")
        else:
            assert torch.equal(last[b], state[b]) and torch.equal(left[b], taps[b])


def test_offsets_outside_the_frames_are_taken_as_the_nearest():
    x, o = scan_inputs(50, 3, 16, 8, 1, "fp32", packed=True)
    w = randn(11, 16, 3)
    good, bad = (torch.tensor(v, dtype=torch.int64, device=DEV) for v in ([0, 20, 50, 50], [-7, 20, 50 + (1 << 40), 1 << 62]))
    for call in (lambda f: sr.selective_scan_run(**x, **o, offsets=f), lambda f: sr.causal_conv_run(x["u"], w, offsets=f)):
        for a, b in zip(call(good), call(bad)):
            assert torch.equal(a, b)


def test_inputs_that_strides_repeat():
    T, B, C, N = 40, 3, 32, 16
    x, o = scan_inputs(T, B, C, N, 1, "bf16")
    x = {k: v if k == "a" else v[:, :1].expand(T, B, *v.shape[2:]) for k, v in x.items()}
    x["b"] = x["b"][:1].expand(T, B, 1, N)
    whole = {k: v.contiguous() for k, v in x.items()}
    z = o["z"][:1].expand(T, B, C)
    for a, b in zip(sr.selective_scan_run(**x, **dict(o, z=z)), sr.selective_scan_run(**whole, **dict(o, z=z.contiguous()))):
        assert torch.equal(a, b)
    w = randn(11, C, 4)
    for a, b in zip(sr.causal_conv_run(x["u"], w), sr.causal_conv_run(whole["u"], w)):
        assert torch.equal(a, b)
    first = {k: v if k == "a" else v[0] for k, v in x.items()}
    s1, s2 = randn(9, B, C, N), randn(9, B, C, N)
    assert torch.equal(sr.selective_scan_step(*first.values(), s1, **dict(o, z=z[0])), sr.selective_scan_step(*(v.contiguous() for v in first.values()), s2, **dict(o, z=z[0])))
    assert torch.equal(s1, s2)


def test_nothing_to_do():
    x, o = scan_inputs(4, 2, 8, 4, 1, "fp32")
    none = {k: v if k == "a" else v[:0] for k, v in x.items()}
    state = randn(9, 2, 8, 4)
    out, last = sr.selective_scan_run(**none, d=o["d"], state=state)
    assert out.shape == (0, 2, 8) and torch.equal(last, state)
    assert not sr.selective_scan_run(**none)[1].any()
    w = randn(11, 8, 4)
    taps = randn(10, 2, 3, 8)
    out, last = sr.causal_conv_run(none["u"], w, state=taps)
    assert out.shape == (0, 2, 8) and torch.equal(last, taps) and not sr.causal_conv_run(none["u"], w)[1].any()
    nobody = {k: v if k == "a" else v[:, :0] for k, v in x.items()}
    assert sr.selective_scan_run(**nobody)[0].shape == (4, 0, 8) and sr.causal_conv_run(nobody["u"], w)[1].shape == (0, 3, 8)
    assert sr.selective_scan_step(*(v if k == "a" else v[0] for k, v in nobody.items()), randn(9, 0, 8, 4)).shape == (0, 8)
    assert sr.block_norm(x["u"][:0, 0], x["dt"][:0, 0])[0].shape == (0, 8)


def test_what_is_written_in_place_gets_a_new_version():
    x, o = scan_inputs(4, 2, 8, 4, 1, "fp32")
    w, state, taps, out = randn(11, 8, 4), randn(9, 2, 8, 4), randn(10, 2, 3, 8), torch.empty(4, 2, 8, device=DEV)
    before = [t._version for t in (state, taps, out)]
    sr.selective_scan_run(**x, state_out=state, out=out)
    sr.causal_conv_step(x["u"][0], w, taps)
    assert [t._version for t in (state, taps, out)] == [v + 1 for v in before]


# ------------------------------------------------------------------------------------------ refusals that need a device
def test_refusals():
    x, o = scan_inputs(6, 2, 8, 4, 2, "fp32")
    w, state = randn(11, 8, 4), randn(9, 2, 8, 4)
    taps = randn(10, 2, 3, 8)
    bad = [
        lambda: sr.selective_scan_run(**dict(x, dt=x["dt"].bfloat16())), lambda: sr.selective_scan_run(**dict(x, dt=x["dt"][:5])), lambda: sr.selective_scan_run(**dict(x, u=x["u"][..., :7])),
        lambda: sr.selective_scan_run(**dict(x, a=x["a"].bfloat16())), lambda: sr.selective_scan_run(**dict(x, a=x["a"].t().contiguous().t())),
        lambda: sr.selective_scan_run(**dict(x, c=x["c"][..., :3])), lambda: sr.selective_scan_run(**dict(x, b=x["b"][:, :, :1])), lambda: sr.selective_scan_run(**dict(x, dt=None)),
        lambda: sr.selective_scan_run(**x, d=o["d"][:7]), lambda: sr.selective_scan_run(**x, z=o["z"][:, :1]), lambda: sr.selective_scan_run(**x, state=state[:1]),
        lambda: sr.selective_scan_run(**x, state=state.double()), lambda: sr.selective_scan_run(**x, out=torch.empty(6, 2, 9, device=DEV)), lambda: sr.selective_scan_run(**x, out=x["dt"]),
        lambda: sr.selective_scan_run(**x, offsets=torch.zeros(3, dtype=torch.int64, device=DEV)), lambda: sr.selective_scan_run(**{k: v if k == "a" else v.half() for k, v in x.items()}),
        lambda: sr.selective_scan_run(**dict(x, u=x["u"].transpose(0, 2).contiguous().transpose(0, 2))), lambda: sr.selective_scan_run(**dict(x, u=x["u"].cpu())),
        lambda: sr.selective_scan_step(x["u"], x["dt"][0], x["a"], x["b"][0], x["c"][0], state), lambda: sr.selective_scan_step(x["u"][0], x["dt"][0], x["a"], x["b"][0], x["c"][0], None),
        lambda: sr.causal_conv_run(x["u"], w[:7]), lambda: sr.causal_conv_run(x["u"], randn(1, 8, 9)), lambda: sr.causal_conv_run(x["u"], w, bias=randn(1, 7)),
        lambda: sr.causal_conv_run(x["u"], w, state=taps.bfloat16()), lambda: sr.causal_conv_run(x["u"], w, state=taps[:, :2]), lambda: sr.causal_conv_step(x["u"][0], w, taps[:, :2]),
        lambda: sr.causal_conv_step(x["u"][0], w, None), lambda: sr.causal_conv_run(x["u"][0], w),
        lambda: sr.block_norm(x["u"][0], x["dt"][1][:1]), lambda: sr.block_norm(x["u"][0], x["dt"][0].bfloat16()), lambda: sr.block_norm(x["u"][0], None),
        lambda: sr.block_norm(x["u"][0], x["dt"][0], gate=x["dt"][0][:, :7]), lambda: sr.block_norm(x["u"][0], x["dt"][0], weight_after=randn(1, 7)),
        lambda: sr.block_norm(x["u"][0], x["dt"][0], norms="all"), lambda: sr.block_norm(x["u"][0], x["dt"][0], gate_act="tanh"), lambda: sr.block_norm(x["u"][0], x["dt"][0], format="mx6"),
        lambda: sr.block_norm(x["u"][0], x["dt"][0], norms="after", format="mx8"), lambda: sr.block_norm(x["u"][0], x["dt"][0], eps=-1.0),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(sr.SrError):
            call()
            pytest.fail("call %d was taken" % k)
    many = scan_inputs(2, 1, 2, 129, 1, "fp32")[0]
    with pytest.raises(sr.SrError):
        sr.selective_scan_run(**many)


# ------------------------------------------------------------------------------------------ norms around a block
def check_block(y, r, after, before, gate, act, scale, eps, norms, out, h, dtype):
    want, wh, mag = oracle.block(host(y), host(r), *(None if t is None else host(t) for t in (after, before, gate)), act, scale, eps, norms)
    n = y.shape[1]
    e = (n ** 0.5 + 16) * 2.0 ** -23 + (2.0 ** -21 if dtype == "fp32" else 2.0 ** -18)           # (sums of n squares, in any order by pairs or threads; the gate)
    within(host(h), wh, oracle.HALF_STEP[dtype] * np.abs(wh) + e * mag, "h")
    if out is not None:
        # an error of h goes through the norm divided by its root mean square, times the weight
        root = np.sqrt((wh * wh).mean(-1, keepdims=True) + eps)
        w = np.abs(host(before)) if before is not None else 1.0
        carried = (e * mag + e * np.abs(wh) * (mag * np.abs(wh)).mean(-1, keepdims=True) / root ** 2) / root * w
        within(host(out), want, oracle.HALF_STEP[dtype] * np.abs(want) + 1.01 * carried + e * np.abs(want), "out")


BLOCKS = [(1, 1), (3, 8), (5, 33), (4, 64), (2, 1000), (7, 1024), (9, 2048), (3, 2050), (2, 4097), (1, 8192), (2, 8200), (1, 16400), (1, 20001)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", BLOCKS)
def test_block_norm(rows, cols, dtype):
    y, r = randn(1, rows, cols, dtype=dtype), randn(2, rows, cols, dtype=dtype)
    gate = randn(3, rows, 2 * cols + 3, dtype=dtype)[:, 3:3 + cols]
    after, before = 1 + 0.2 * randn(4, cols), 1 + 0.2 * randn(5, cols)
    for norms in ("both", "after", "before", "none"):
        for g, act in ((gate, "sigmoid"), (None, "none"), (gate, "silu"), (r[:1].expand(rows, cols), "none")):
            got = sr.block_norm(y, r, after, before, gate=g, gate_act=act, scale=0.7, eps=1e-5, norms=norms)
            out, h = got if norms in ("both", "before") else (None, got)
            check_block(y, r, after, before, g, act, 0.7, 1e-5, norms, out, h, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("format", ["mx4", "mx8"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (5, 100), (130, 256), (3, 1003), (2, 9000), (1, 20001)])
def test_block_norm_microscaled(rows, cols, format, dtype):
    y, r, gate = (randn(k, rows, cols, dtype=dtype) for k in (1, 2, 3))
    m, h = sr.block_norm(y, r, gate=gate, scale=0.5, format=format)
    assert torch.equal(h, sr.block_norm(y, r, gate=gate, scale=0.5)[1])
    # the elements are rounded from 32-bit values.  4 bits, scale s: off by s beyond 4 s, which only a group whose largest value g is more has (s < g / 4), by s / 2 below (s < g / 3);
    # 8 bits: half a step, or half of the smallest one, 2^-10 s, s < g / 224
    want, _, _ = oracle.block(host(y), host(r), gate=host(gate), scale=0.5)
    groups = np.pad(np.abs(want), ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32).max(-1).repeat(32, -1)[:, :cols]
    bound = 0.25 * groups if format == "mx4" else 2.0 ** -4 * np.abs(want) + 2.0 ** -15 * groups
    within(host(m.values()), want, bound * 1.001 + 1e-5 * groups)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [64, 100, 9000])
def test_block_norm_rows_out_of_range(cols, dtype):
    y, r = randn(1, 6, cols, dtype=dtype), randn(2, 6, cols, dtype=dtype)
    big = torch.tensor([1e30, 1e-30, 1e20, 1.0, 1e-20, 1e36], device=DEV).to(DT[dtype])[:, None]
    out, h = sr.block_norm(y * big, r * big, eps=0.0)
    check_block(y * big, r * big, None, None, None, "none", 1.0, 0.0, "both", out, h, dtype)
    zero = torch.zeros_like(y)
    out, h = sr.block_norm(zero, r)
    assert torch.equal(h, r)
    out, h = sr.block_norm(zero, zero)
    assert torch.equal(out, zero) and torch.equal(h, zero)


def test_block_norm_what_is_not_finite_stays_in_its_row():
    y, r, gate = (randn(k, 9, 200) for k in (1, 2, 3))
    out, h = sr.block_norm(y, r, gate=gate)
    for t in (y, r, gate):
        kept = t[4, 11].clone()
        for value in (float("inf"), float("nan")):
            t[4, 11] = value
            o, g = sr.block_norm(y, r, gate=gate)
            rows = torch.arange(9, device=DEV) != 4
            assert torch.equal(o[rows], out[rows]) and torch.equal(g[rows], h[rows])
        t[4, 11] = kept


# ------------------------------------------------------------------------------------------ the head
def head_weights(channels, inner, states, rank, width, groups, outputs, blocks, seed=0):
    rng = np.random.default_rng(seed)

    def mat(rows, cols):
        return torch.tensor(rng.standard_normal((rows, cols)) / np.sqrt(cols), dtype=torch.float32)

    def vec(n, mean=0.0, dev=0.1):
        return torch.tensor(mean + dev * rng.standard_normal(n), dtype=torch.float32)

    return {"blocks": [{"norm": vec(channels, 1.0), "in": mat(2 * inner + channels, channels), "conv": mat(inner, width), "conv_bias": vec(inner),
                        "x": mat(rank + 2 * groups * states, inner), "dt": mat(inner, rank), "dt_bias": vec(inner, -3.0, 1.0),
                        "a": -torch.arange(1, states + 1).float().repeat(inner, 1), "d": vec(inner, 1.0), "o": mat(channels, inner), "norm_after": vec(channels, 1.0)}
                       for _ in range(blocks)],
            "norm_out": vec(channels, 1.0), "out": mat(outputs, channels), "bias": vec(outputs)}


def head_oracle(w, x, inner, states, rank, groups, fmt, scale, eps):
    """x [T][B][channels] through the head in 64 bits, operands of products rounded to the format."""
    def lin(x, m):
        return operator_oracle.quantize(x, fmt)[2] @ operator_oracle.quantize(np.asarray(m, np.float64), fmt)[2].T

    T, B, C = x.shape
    h = x.reshape(T * B, C)
    m = oracle.rms(h, w["blocks"][0]["norm"], eps)
    for i, k in enumerate(w["blocks"]):
        p = lin(m, k["in"]).reshape(T, B, -1)
        y = np.zeros((T, B, inner))
        u = np.stack([oracle.conv(p[:, b, :inner], k["conv"], k["conv_bias"], True)[0] for b in range(B)], 1)
        low = lin(u.reshape(T * B, inner), k["x"])
        dt = lin(low[:, :rank], k["dt"]).reshape(T, B, inner)
        bc = low[:, rank:].reshape(T, B, 2, groups, states)
        for b in range(B):
            y[:, b] = oracle.scan(u[:, b], dt[:, b], k["a"], bc[:, b, 0], bc[:, b, 1], k["d"], p[:, b, inner:2 * inner], k["dt_bias"])[0]
        o = lin(y.reshape(T * B, inner), k["o"])
        before = w["blocks"][i + 1]["norm"] if i + 1 < len(w["blocks"]) else w["norm_out"]
        m, h, _ = oracle.block(o, h, k["norm_after"], before, p[..., 2 * inner:].reshape(T * B, -1), "sigmoid", scale, eps)
    return (lin(m, w["out"]) + np.asarray(w["bias"], np.float64)).reshape(T, B, -1)


@pytest.mark.parametrize("fmt,blocks,groups", [("mx8", 1, 1), ("mx8", 2, 2), ("mx4", 1, 1)])
def test_head_runs_steps_and_captures(fmt, blocks, groups):
    C, inner, N, rank, W, T, B, outs = 64, 96, 16, 4, 4, 12, 3, 10
    w = head_weights(C, inner, N, rank, W, groups, outs, blocks)
    head = sr.SelectiveHead(w, C, inner, N, rank, W, B, groups=groups, scale=0.5, format=fmt, dtype="fp32", eps=1e-6)
    x = randn(1, T, B, C)
    run = head.run(x)
    want = head_oracle(w, host(x), inner, N, rank, groups, fmt, 0.5, 1e-6)
    # a value that lies next to a border of the format may be rounded to the other side: a few operands of products differ by a step
    scale = np.sqrt((want ** 2).mean())
    assert np.sqrt(((host(run) - want) ** 2).mean()) <= (0.02 if fmt == "mx8" else 0.1) * scale
    after = head.get_state()
    head.reset()
    steps = torch.stack([head.step(x[t]) for t in range(T)])
    assert (steps - run).square().mean().sqrt() <= (0.02 if fmt == "mx8" else 0.1) * scale
    # two halves are the whole, and a state can be put back
    head.reset()
    first = head.run(x[:5])
    middle = head.get_state()
    second = head.run(x[5:])
    assert (torch.cat((first, second)) - run).square().mean().sqrt() <= (0.02 if fmt == "mx8" else 0.1) * scale
    head.set_state(middle)
    assert torch.equal(head.run(x[5:]), second)
    # captured once, replayed with other features
    frame = x[0].clone()
    head.reset()
    head.step(frame)
    head.reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head.step(frame)
    head.reset()
    for t in range(T):
        frame.copy_(x[t])
        graph.replay()
        assert torch.equal(out, steps[t]), t
    assert all(torch.isfinite(s).all() for pair in after for s in pair)
    sr.operator_status(DEV)


def test_head_behind_a_rollout():
    from workloads import data, graphs
    spec = graphs.build("c2", batch=4, frames=3)
    X, Wt, Bi = data.make_inputs(spec), data.make_weights(spec), data.make_biases(spec)
    G = sr.Graph(spec.nodes, spec.edges, spec.patterns["streaming"], batch=spec.batch, dtype=spec.dtype)
    G.set_weights(Wt, Bi)
    frames = [torch.from_numpy(X[v]).to(DEV).to(DT[spec.dtype]).contiguous() for v in G.input_nodes]
    features = G.rollout(frames)
    channels = features[0, 0].numel()
    w = head_weights(channels, 64, 8, 4, 3, 1, 5, 2)
    head = sr.SelectiveHead(w, channels, 64, 8, 4, 3, spec.batch, format="mx8", dtype="fp32")
    out = G.rollout(frames, head=head)
    head.reset()
    assert torch.equal(out, head.run(features)) and out.shape == (features.shape[0], 4, 5)
    with pytest.raises(sr.SrError):
        G.rollout(frames, head=sr.SelectiveHead(w, channels, 64, 8, 4, 3, spec.batch + 1, format="mx8", dtype="fp32"))


# ------------------------------------------------------------------------------------------ streams, threads
def test_calls_of_two_threads():
    import threading
    x, o = scan_inputs(200, 2, 32, 16, 1, "bf16")
    w = randn(7, 32, 4)
    y = [randn(30 + k, 400, 520, dtype="bf16") for k in range(3)]
    calls = (lambda: sr.selective_scan_run(**x, **o), lambda: sr.causal_conv_run(x["u"], w, silu=True), lambda: sr.block_norm(*y[:2], gate=y[2]))
    want = [f() for f in calls]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = [calls[(k + j) % 3]() for j in range(30)]
            torch.cuda.current_stream().synchronize()
            wrong.extend(j for j, g in enumerate(got) if not all(torch.equal(a, b) for a, b in zip(g, want[(k + j) % 3])))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not wrong


def test_block_norm_goes_over_many_rows():
    """More rows than blocks, so that blocks go over several."""
    for rows, cols, norms in ((6000, 40, "both"), (5001, 1030, "after"), (3000, 2048, "before"), (2500, 999, "both")):
        y, r, gate = (randn(k, rows, cols, dtype="bf16") for k in (1, 2, 3))
        got = sr.block_norm(y, r, gate=gate, scale=0.5, norms=norms)
        out, h = got if norms in ("both", "before") else (None, got)
        check_block(y, r, None, None, gate, "sigmoid", 0.5, 1e-6, norms, out, h, "bf16")


def test_calls_side_by_side_on_streams_and_replayed():
    x, o = scan_inputs(400, 1, 64, 16, 1, "bf16")
    y, p = scan_inputs(300, 2, 64, 16, 1, "bf16", seed=20)
    w = randn(7, 64, 4)
    want = [sr.selective_scan_run(**x, **o), sr.selective_scan_run(**y, **p), sr.causal_conv_run(x["u"], w, silu=True)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, f in zip(streams, (lambda: sr.selective_scan_run(**x, **o), lambda: sr.selective_scan_run(**y, **p), lambda: sr.causal_conv_run(x["u"], w, silu=True))):
            with torch.cuda.stream(s):
                got.append(f())
    torch.cuda.synchronize()
    for k, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[k % 3]))
    graphs = []
    for f in (lambda: sr.selective_scan_run(**x, **o), lambda: sr.selective_scan_run(**y, **p)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = f()
        graphs.append((g, res))
    for _ in range(2):
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for k, (_, res) in enumerate(graphs):
        assert all(torch.equal(a, b) for a, b in zip(res, want[k]))
