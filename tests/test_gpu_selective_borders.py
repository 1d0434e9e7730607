"""The selective head's operators where they can go wrong: what is not finite, frame by frame and in runs."""
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import selective

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
DEV = "cuda:0"
NAN = float("nan")


def randn(seed, *shape, dtype="fp32"):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).to(DEV)


def inputs(lead, channels, states, groups, dtype, gap=0, seed=0):
    """gap: elements ahead of b in the rows that b and c are taken from."""
    low = randn(seed + 1, *lead, gap + 2 * groups * states, dtype=dtype)
    b, c = (low[..., gap + k * groups * states:gap + (k + 1) * groups * states].unflatten(-1, (groups, states)) for k in (0, 1))
    a = -torch.arange(1, states + 1, device=DEV).float() * torch.exp(0.2 * randn(seed + 3, channels, states))
    return dict(u=randn(seed + 2, *lead, channels, dtype=dtype), dt=randn(seed + 4, *lead, channels, dtype=dtype), a=a.contiguous(), b=b, c=c,
                d=randn(seed + 5, channels), z=randn(seed + 7, *lead, channels, dtype=dtype), dt_bias=randn(seed + 6, channels) - 3.0)


# ------------------------------------------------------------------------------------------ what is not finite
# What is NaN: where in the tensor, and what of the states [sequences][channels][states] and outputs [sequences][channels] is NaN then.  (Two groups of channels, channel 3 in the first.)
def reaches(what, batch, channels, states):
    h = torch.zeros(batch, channels, states, dtype=torch.bool, device=DEV)
    y = torch.zeros(batch, channels, dtype=torch.bool, device=DEV)
    half = channels // 2
    place = {"a": (3, 1), "u": (1, 3), "dt": (1, 3), "z": (1, 3), "b": (1, 0, 1), "c": (1, 0, 1), "d": (3,), "dt_bias": (3,), "state": (1, 3, 1)}[what]
    if what == "a":
        h[:, 3, 1] = True
    elif what in ("u", "dt"):
        h[1, 3] = True
    elif what == "dt_bias":
        h[:, 3] = True
    elif what == "b":
        h[1, :half, 1] = True
    elif what == "state":
        h[1, 3, 1] = True
    elif what == "c":
        y[1, :half] = True
    elif what == "z":
        y[1, 3] = True
    else:
        y[:, 3] = True
    return place, h, y | h.any(-1)


NOT_FINITE = ["a", "u", "dt", "z", "b", "c", "d", "dt_bias", "state"]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("batch,states,gap", [(2, 16, 0), (20, 16, 0), (3, 5, 3), (4, 20, 5), (3, 100, 1), (2, 128, 0)])
@pytest.mark.parametrize("what", NOT_FINITE)
def test_single_frames_keep_what_is_not_a_number(what, batch, states, gap, dtype):
    channels = 12
    place, bad_h, bad_y = reaches(what, batch, channels, states)
    for entering in (torch.zeros(batch, channels, states, device=DEV), randn(9, batch, channels, states)):
        x = inputs((batch,), channels, states, 2, dtype, gap)
        clean = entering.clone()
        want = sr.selective_scan_step(state=clean, **x)
        state = entering.clone()
        dict(x, state=state)[what][place] = NAN
        _, run = sr.selective_scan_run(**{k: v if k in ("a", "d", "dt_bias") else v[None] for k, v in x.items()}, state=state.clone())
        out = sr.selective_scan_step(state=state, **x)
        assert torch.equal(torch.isnan(state), bad_h) and torch.equal(torch.isnan(out), bad_y) and torch.equal(torch.isnan(run), bad_h)
        assert torch.equal(state[~bad_h], clean[~bad_h]) and torch.equal(out[~bad_y], want[~bad_y])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("frames,states", [(40, 16), (40, 5), (333, 12), (333, 32), (333, 128)])
@pytest.mark.parametrize("what", ["a", "d", "dt_bias", "state"])
def test_runs_keep_what_is_not_a_number(what, frames, states, dtype):
    channels, batch = 12, 2
    assert (selective.scan_plan(DT[dtype], batch, frames, channels, states, 2)["segment"] > 0) == (frames > 40)
    place, bad_h, bad_y = reaches(what, batch, channels, states)
    for entering in (torch.zeros(batch, channels, states, device=DEV), randn(9, batch, channels, states)):
        x = inputs((frames, batch), channels, states, 2, dtype)
        want, clean = sr.selective_scan_run(state=entering, **x)
        state = entering.clone()
        dict(x, state=state)[what][place] = NAN
        out, last = sr.selective_scan_run(state=state, **x)
        assert torch.equal(torch.isnan(last), bad_h) and torch.equal(torch.isnan(out), bad_y.expand_as(out))
        assert torch.equal(last[~bad_h], clean[~bad_h]) and torch.equal(out[:, ~bad_y], want[:, ~bad_y])


# ------------------------------------------------------------------------------------------ many packed sequences
@pytest.mark.parametrize("longest", [2000, 3], ids=["one_long", "none_long"])
def test_packed_sequences_more_than_a_launch_has_rows(longest):
    """More than 65535, the long one among the last; and in a time that grows with the sequences, not with their square (70000 of them, each looked at by a block for each: seconds)."""
    import numpy as np
    from tests.test_gpu_selective import check_scan, spans
    rng = np.random.default_rng(7)
    B, C, N = 70000, 8, 4
    lengths = rng.integers(0, 4, B)
    lengths[66001] = longest
    at, offsets = spans(lengths)
    total = int(at[-1])
    assert selective.scan_plan(torch.float32, B, total, C, N, 1, packed=True)["segment"] > 0
    x = inputs((total,), C, N, 1, "fp32")
    o = {k: x.pop(k) for k in ("d", "z", "dt_bias")}
    state = randn(9, B, C, N)
    entering = state.clone()
    sr.selective_scan_run(**x, **o, state=state, offsets=offsets)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out, last = sr.selective_scan_run(**x, **o, state=state, offsets=offsets, state_out=state)
    end.record()
    end.synchronize()
    assert begin.elapsed_time(end) < 30.0
    for b in [0, 1, 2, *range(3, B, 3511), 65534, 65535, 65536, 66000, 66001, 66002, B - 1]:
        s = slice(at[b], at[b + 1])
        if lengths[b]:
            check_scan({k: v if k == "a" else v[s] for k, v in x.items()}, dict(o, z=o["z"][s]), True, entering[b], out[s], last[b], b, "fp32")
        else:
            assert torch.equal(last[b], entering[b])


def test_packed_sequences_captured_with_other_lengths():
    """The sizes say how a run is cut; what is long is found when it is replayed."""
    from tests.test_gpu_selective import check_scan
    B, T, C, N = 300, 1200, 8, 4
    x = inputs((T,), C, N, 1, "fp32")
    o = {k: x.pop(k) for k in ("d", "z", "dt_bias")}
    state = randn(9, B, C, N)
    offsets = torch.arange(B + 1, device=DEV) * 4
    assert selective.scan_plan(torch.float32, B, T, C, N, packed=True)["segment"] > 0
    sr.selective_scan_run(**x, **o, state=state, offsets=offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, last = sr.selective_scan_run(**x, **o, state=state, offsets=offsets)
    one_long = torch.full((B,), 2, device=DEV)
    one_long[211] = T - 2 * (B - 1)
    for lengths in (torch.full((B,), 4, device=DEV), one_long, torch.full((B,), 4, device=DEV)):
        offsets[1:] = lengths.cumsum(0)
        out.fill_(float("nan"))
        graph.replay()
        at = offsets.tolist()
        assert torch.isfinite(out).all()
        for b in (0, 1, 210, 211, 212, 299):
            s = slice(at[b], at[b + 1])
            check_scan({k: v if k == "a" else v[s] for k, v in x.items()}, dict(o, z=o["z"][s]), True, state[b], out[s], last[b], b, "fp32")


# ------------------------------------------------------------------------------------------ sizes
def test_places_beyond_32_bits():
    """More than 2^31 elements: the last frames, or sequences, are those of a call on them alone."""
    T, C, W, tail = 1 << 19, 4104, 4, 3000
    x = torch.empty(T, 1, C, dtype=torch.bfloat16, device=DEV)
    x.view(-1, 64, C)[:] = randn(1, 64, C, dtype="bf16")
    x[-tail:] = randn(2, tail, 1, C, dtype="bf16")
    assert x.numel() > 1 << 31
    w = randn(3, C, W)
    out, last = sr.causal_conv_run(x, w, silu=True)
    part, left = sr.causal_conv_run(x[-tail - 3:], w, silu=True)
    assert torch.equal(out[-tail:], part[3:]) and torch.equal(last, left)
    del out
    # states that lose two thirds of themselves in a frame at least: 200 frames later nothing is left of what came before
    a, bc, dt = -1.0 - torch.rand(C, 4, device=DEV), randn(4, 1, 1, 1, 4, dtype="bf16").expand(T, 1, 1, 4), torch.ones(1, 1, C, dtype=torch.bfloat16, device=DEV).expand(T, 1, C)
    out, last = sr.selective_scan_run(x, dt, a, bc, bc, softplus=False)
    part, left = sr.selective_scan_run(x[-tail:], dt[-tail:], a, bc[-tail:], bc[-tail:], softplus=False)
    # (a step of bf16 between two roundings of nearly the same value)
    torch.testing.assert_close(out[-tail + 200:].float(), part[200:].float(), rtol=2.0 ** -7, atol=1e-4)
    torch.testing.assert_close(last, left, rtol=1e-4, atol=1e-5)
    del out
    y = x.view(T, C)
    h, g = sr.block_norm(y, y, gate=y, norms="both")
    ph, pg = sr.block_norm(y[-tail:], y[-tail:], gate=y[-tail:], norms="both")
    assert torch.equal(h[-tail:], ph) and torch.equal(g[-tail:], pg)
    del h, g
    taps = torch.zeros(T, 1, C, dtype=torch.bfloat16, device=DEV)
    taps[-tail:, 0] = y[:tail]
    some = taps[-tail:].clone()
    out = sr.causal_conv_step(y, w[:, :2].contiguous(), taps)
    assert torch.equal(out[-tail:], sr.causal_conv_step(y[-tail:], w[:, :2].contiguous(), some)) and torch.equal(taps[-tail:], some)
    del out, taps
    state = torch.zeros(T, C, 1, device=DEV)
    state[-tail:, :, 0] = y[:tail].float()
    some = state[-tail:].clone()
    args = lambda n: (dt[:n, 0].expand(n, C), a[:, :1].contiguous(), bc[:n, 0, :, :1], bc[:n, 0, :, :1])
    out = sr.selective_scan_step(y, *args(T), state, softplus=False)
    assert torch.equal(out[-tail:], sr.selective_scan_step(y[-tail:], *args(tail), some, softplus=False)) and torch.equal(state[-tail:], some)


def test_more_sequences_than_32_bits_count_are_refused():
    many = (1 << 32) + 5
    x, w, a = torch.zeros(1, 1, 1, device=DEV).expand(1, many, 1), torch.zeros(1, 1, device=DEV), torch.zeros(1, 1, device=DEV)
    bc = x[..., None]
    for call in (lambda: sr.causal_conv_run(x, w, out=None), lambda: sr.selective_scan_run(x, x, a, bc, bc), lambda: sr.causal_conv_run(x[:, :(1 << 31) - 1], w)):
        with pytest.raises(sr.SrError):
            call()
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------ heads
def heads():
    from tests.test_gpu_selective import head_weights
    from tests.test_operator_refusals import weights
    return lambda batch: sr.SelectiveHead(head_weights(32, 32, 8, 2, 4, 1, 3, 1), 32, 32, 8, 2, 4, batch), lambda batch: sr.TemporalHead(weights(channels=32), 32, 4, 2, 32, 48, batch)


@pytest.mark.parametrize("kind", [0, 1], ids=["selective", "temporal"])
def test_heads_of_no_frames_and_of_no_sequences(kind):
    make = heads()[kind]
    head = make(2)
    x = randn(1, 5, 2, 32)
    one = head.run(x)
    head.reset()
    parts = [head.run(x[:0]), head.run(x[:3]), head.run(x[3:3]), head.run(x[3:])]
    assert [tuple(p.shape) for p in parts] == [(n, 2, head.outputs) for n in (0, 3, 0, 2)]
    torch.testing.assert_close(torch.cat(parts), one, rtol=0.1, atol=0.1 * float(one.abs().max()))
    nobody = make(0)
    assert nobody.run(x[:, :0]).shape == (5, 0, head.outputs) and nobody.step(x[0, :0]).shape == (0, head.outputs)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", [0, 1], ids=["selective", "temporal"])
def test_heads_refuse_what_is_no_tensor(kind):
    import numpy as np
    head = heads()[kind](2)
    x = randn(1, 5, 2, 32)
    one = head.run(x)
    head.reset()
    for no in (None, 3, "x", [1.0], np.zeros((5, 2, 32), np.float32), [None], [(None, None)], [(3, 4)], {}):
        for call in (head.run, head.step, head.set_state):
            with pytest.raises(sr.SrError):
                call(no)
    assert torch.equal(head.run(x), one)
