"""The temporal head's operators on the GPU where their paths meet: precision, borders of segments and tiles, rows at the ends of the range.

Bounds as in test_gpu_operators.py; where they are tighter the test says why."""
import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from tests import operator_oracle as oracle
from tests.test_gpu_operators import DEV, TYPES, gen, host, inputs, within
from tests.test_operator_plans import PRODUCTS, RUNS, plan

pytestmark = pytest.mark.gpu


def compare(q, k, v, d, state, out, last, scale, dtype, sequences):
    """Outputs within half a step of their type and what sums in 32 bits lose; factors that bf16 runs hold in two bf16 parts (the weights of a
    chunk's frames, the state) leave 2^-16 of a term's magnitude, and one of the two enters each term: 2^-15 covers both."""
    for b, at in enumerate(sequences):
        n = q[at].shape[0]
        dd = host(d if d.dim() == 1 else d[at])
        want, S, mag, A = oracle.attention(host(q[at]), host(k[at]), host(v[at]), dd, None if state is None else host(state[b]), scale)
        steps = (2 * n + q.shape[-1] + 40) * 2.0 ** -23
        parts = 2.0 ** -15 if dtype == "bf16" else 0.0
        if n:
            within(out[at], want, oracle.HALF_STEP[dtype] * np.abs(want) + (steps + parts) * mag)
        within(last[b], S, steps * A)


# ------------------------------------------------------------------------------------------ precision of bf16 runs
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T, B, heads, groups, dk, dv", [(16, 1, 1, 1, 64, 64), (100, 2, 2, 2, 128, 128), (129, 2, 4, 2, 64, 64), (200, 1, 3, 3, 40, 72), (257, 2, 4, 1, 128, 64),
                                                         (130, 1, 2, 2, 96, 200), (2500, 1, 2, 1, 64, 64)])
def test_bf16_runs_are_as_exact_as_their_outputs(T, B, heads, groups, dk, dv, gated):
    q, k, v, d = inputs((T, B), heads, groups, dk, dv, "bf16", gated, seed=90)
    state = torch.randn(B, groups, dk, dv, generator=gen(91), device=DEV)
    out, last = sr.linear_attention_run(q, k, v, d, state=state, scale=0.3)
    compare(q, k, v, d, state, out, last, 0.3, "bf16", [(slice(None), b) for b in range(B)])


# ------------------------------------------------------------------------------------------ segments
def offsets_of(lengths):
    first = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    return torch.tensor(first, dtype=torch.int64, device=DEV), [slice(a, b) for a, b in zip(first, first[1:])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lengths, heads, groups, dk, dv, segment", RUNS)
def test_packed_sequences_that_are_cut(lengths, heads, groups, dk, dv, segment, dtype):
    spare, total = 40, sum(lengths)
    p = sr.operators.attention_plan(TYPES[dtype], len(lengths), total + spare, heads, groups, dk, dv, packed=True)
    assert p["segment"] > 0 and p["chunk"] == (128 if dtype == "bf16" else 16)
    q, k, v, d = inputs((total + spare,), heads, groups, dk, dv, dtype, True, seed=100)
    d = d / 50                                                  # (memories of hundreds of frames: what goes from segment to segment matters)
    for t in (q, k, v):
        t[total:] = float("nan")
    offsets, at = offsets_of(lengths)
    state = torch.randn(len(lengths), groups, dk, dv, generator=gen(101), device=DEV)
    out = torch.full((total + spare, heads, dv), 5.0, dtype=TYPES[dtype], device=DEV)
    _, last = sr.linear_attention_run(q, k, v, d, state=state, offsets=offsets, scale=0.5, out=out)
    compare(q, k, v, d, state, out, last, 0.5, dtype, at)
    assert (out[total:] == 5).all()
    for b, n in enumerate(lengths):
        if n == 0:
            assert torch.equal(last[b], state[b])
    kept = state.clone()
    sr.linear_attention_run(q, k, v, d, state=kept, offsets=offsets, scale=0.5, out=out, state_out=kept)
    assert torch.equal(kept, last)
    sr.operator_status()


@pytest.mark.parametrize("T, B, heads, groups, dk, dv", [(5000, 1, 4, 1, 64, 64), (3001, 2, 4, 2, 128, 128), (4097, 1, 6, 3, 40, 72)])
def test_cut_runs_with_heads_that_share_a_state(T, B, heads, groups, dk, dv):
    assert sr.operators.attention_plan(torch.bfloat16, B, T, heads, groups, dk, dv)["segment"] > 0
    q, k, v, d = inputs((T, B), heads, groups, dk, dv, "bf16", True, seed=102)
    d = d / 50
    state = torch.randn(B, groups, dk, dv, generator=gen(103), device=DEV)
    out, last = sr.linear_attention_run(q, k, v, d, state=state, scale=0.3)
    compare(q, k, v, d, state, out, last, 0.3, "bf16", [(slice(None), b) for b in range(B)])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_states_that_start_anew_at_borders_of_segments(dtype):
    lengths, heads, groups, dk, dv, segment = RUNS[0]
    offsets, at = offsets_of(lengths)
    q, k, v, d = inputs((sum(lengths),), heads, groups, dk, dv, dtype, True, seed=104)
    d = d / 50
    for f in (segment - 1, segment, 2 * segment + 1, 3 * segment + 127, 4 * segment + 128, 5000, 5001, 5000 + segment):
        d[f] = float("-inf")
    d[6 * segment:7 * segment] = -200.0
    state = torch.randn(len(lengths), groups, dk, dv, generator=gen(105), device=DEV)
    out, last = sr.linear_attention_run(q, k, v, d, state=state, offsets=offsets)
    compare(q, k, v, d, state, out, last, 1.0, dtype, at)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("frame", [511, 512, 700, 5002, 5000 + 512])
def test_values_that_are_not_finite_stay_behind_their_frame_across_segments(frame, dtype):
    lengths, heads, groups, dk, dv, segment = RUNS[0]
    offsets, at = offsets_of(lengths)
    q, k, v, d = inputs((sum(lengths),), heads, groups, dk, dv, dtype, True, seed=106)
    d = d / 50
    clean, end = sr.linear_attention_run(q, k, v, d, offsets=offsets)
    v[frame, 0, 5] = float("nan")
    out, last = sr.linear_attention_run(q, k, v, d, offsets=offsets)
    b = next(i for i, s in enumerate(at) if s.start <= frame < s.stop)
    other = [c for c in range(dv) if c != 5]
    assert torch.isnan(out[frame:at[b].stop, :, 5]).all() and torch.isnan(last[b, 0, :, 5]).all()
    assert torch.equal(out[:frame], clean[:frame]) and torch.equal(out[at[b].stop:], clean[at[b].stop:])
    assert torch.equal(out[:, :, other], clean[:, :, other]) and torch.equal(last[:, :, :, other], end[:, :, :, other])
    assert torch.equal(torch.cat((last[:b], last[b + 1:])), torch.cat((end[:b], end[b + 1:])))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T, frame", [(140, 2), (140, 63), (140, 131), (3000, 1027)])
def test_a_decay_that_is_nan_reaches_no_earlier_frame(T, frame, dtype):
    q, k, v, d = inputs((T, 2), 2, 1, 64, 64, dtype, True, seed=107)
    clean, end = sr.linear_attention_run(q, k, v, d)
    d[frame, 0] = float("nan")
    out, last = sr.linear_attention_run(q, k, v, d)
    assert torch.equal(out[:frame], clean[:frame]) and torch.equal(out[:, 1], clean[:, 1]) and torch.equal(last[1], end[1])
    assert torch.isnan(out[frame:, 0]).all() and torch.isnan(last[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T, frame", [(140, 5), (140, 130), (3000, 1500)])
def test_queries_keys_and_states_that_are_not_finite_stay_where_they_are(T, frame, bad, dtype):
    H, G, D = 4, 2, 64                                          # heads 0 and 1 share group 0
    q, k, v, d = inputs((T, 2), H, G, D, D, dtype, True, seed=108)
    state = torch.randn(2, G, D, D, generator=gen(109), device=DEV)
    clean, end = sr.linear_attention_run(q, k, v, d, state=state)
    q2 = q.clone()
    q2[frame, 0, 1, 7] = bad
    out, last = sr.linear_attention_run(q2, k, v, d, state=state)
    touched = torch.zeros(T, 2, H, dtype=torch.bool, device=DEV)
    touched[frame, 0, 1] = True
    assert torch.equal(out[~touched], clean[~touched]) and torch.equal(last, end) and not torch.isfinite(out[frame, 0, 1]).any()
    k2 = k.clone()
    k2[frame, 0, 0, 7] = bad
    out, last = sr.linear_attention_run(q, k2, v, d, state=state)
    touched[frame:, 0, :2] = True
    assert torch.equal(out[~touched], clean[~touched]) and not torch.isfinite(out[frame, 0, :2]).any()
    rows = [i for i in range(D) if i != 7]
    assert torch.equal(last[1], end[1]) and torch.equal(last[0, 1], end[0, 1]) and torch.equal(last[0, 0, rows], end[0, 0, rows])
    state2 = state.clone()
    state2[0, 1, 3, 9] = bad
    out, last = sr.linear_attention_run(q, k, v, d, state=state2)
    columns = [j for j in range(D) if j != 9]
    assert torch.equal(out[:, 1], clean[:, 1]) and torch.equal(out[:, 0, :2], clean[:, 0, :2]) and torch.equal(out[:, 0, 2:][..., columns], clean[:, 0, 2:][..., columns])
    assert torch.equal(last[0, 1][:, columns], end[0, 1][:, columns]) and not torch.isfinite(out[0, 0, 2:, 9]).any()


# ------------------------------------------------------------------------------------------ products
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows, cols, outs, fmt, want", PRODUCTS)
def test_every_way_to_cut_a_product(rows, cols, outs, fmt, want, dtype):
    assert plan(rows, cols, outs, fmt, 0) == want               # on this device
    a = torch.randn(rows, cols, generator=gen(110), device=DEV) * torch.exp(torch.randn(rows, 1, generator=gen(111), device=DEV))
    w = torch.randn(outs, cols, generator=gen(112), device=DEV)
    bias = torch.randn(outs, generator=gen(113), device=DEV)
    qa, qw = sr.quantize(a, fmt), sr.quantize(w, fmt)
    va, vw = qa.values().double(), qw.values().double()
    exact, mag = va @ vw.t() + bias, va.abs() @ vw.abs().t() + bias.abs()
    bound = host(oracle.HALF_STEP[dtype] * exact.abs() + (cols + 1) * 2.0 ** -23 * mag)
    within(sr.product(qa, qw, bias=bias, dtype=TYPES[dtype]), host(exact), bound)
    out = torch.full((rows, outs + 3), 7.0, dtype=TYPES[dtype], device=DEV)
    sr.product(qa, qw, bias=bias, relu=True, out=out[:, :outs])  # rows with gaps
    assert (out[:, outs:] == 7).all()
    within(out[:, :outs], host(exact.clamp_min(0)), bound)
    sr.operator_status()


# ------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows, cols, dtype", [(3, 40959, "bf16"), (9, 40953, "bf16"), (2, 32769, "bf16"), (3, 20479, "fp32"), (5, 20477, "fp32"), (2, 16385, "fp32")])
def test_norm_of_wide_rows_that_start_off_16_bytes(rows, cols, dtype, residual):
    # wider than the registers of 1024 threads hold, the row's last unit behind the last whole pass of them
    x = torch.randn(rows, cols, generator=gen(92), device=DEV).to(TYPES[dtype])
    r = torch.randn(rows, cols, generator=gen(93), device=DEV).to(TYPES[dtype]) if residual else None
    w = torch.randn(cols, generator=gen(94), device=DEV)
    got = sr.rms_norm(x, w, residual=r, eps=1e-5)
    y, s = oracle.norm(host(x), host(w), None if r is None else host(r), 1e-5)
    bound = (oracle.HALF_STEP[dtype] + ((cols + 3) / 2 + 8) * 2.0 ** -23) * np.abs(y)
    if residual:
        bound = bound + 2.0 ** -23 * np.abs(host(w)) * (np.abs(host(x)) + np.abs(host(r))) / np.sqrt((s * s).mean(-1, keepdims=True) + 1e-5)
        within(got[1], s, (oracle.HALF_STEP[dtype] + 2.0 ** -24) * np.abs(s))
        got = got[0]
    within(got, y, bound)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [1, 7, 96, 1003, 4096, 40959])
def test_norm_of_rows_whose_squares_leave_32_bits(cols, dtype):
    sizes = [1e20, 3e38, 2e19, 1e-30, 1e-42, 1e-20, 1.0, 1e19]
    x = torch.empty(len(sizes), cols, device=DEV).uniform_(0.5, 1.0, generator=gen(95)) * torch.tensor(sizes, device=DEV)[:, None]
    x = (x * torch.where(torch.rand(x.shape, generator=gen(96), device=DEV) < 0.5, -1.0, 1.0)).to(TYPES[dtype])
    w = torch.randn(cols, generator=gen(97), device=DEV)
    for eps in (0.0, 1e-12, 1e-30, 1e-44):
        eps = float(np.float32(eps))
        y = oracle.norm(host(x), host(w), eps=eps)[0]
        # as for other rows, and three steps more for the root of eps, its square and the row's division
        bound = (oracle.HALF_STEP[dtype] + ((cols + 3) / 2 + 11) * 2.0 ** -23) * np.abs(y) + 2.0 ** -148
        bound = np.nan_to_num(bound) + (2.0 ** -133 if dtype == "bf16" else 0.0)           # (zeros over zero are NaN on both sides)
        within(sr.rms_norm(x, w, eps=eps), y, bound)
        if dtype == "fp32":
            got = sr.rms_norm(x, w, eps=eps, format="mx8")
            again = sr.quantize(sr.rms_norm(x, w, eps=eps), "mx8")
            assert torch.equal(got.data, again.data) and torch.equal(got.values(), again.values())


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [5, 72, 200, 1000])
def test_padding_is_zero_in_rows_that_are_not_finite(cols, dtype, fmt):
    x = torch.randn(6, cols, generator=gen(98), device=DEV).to(TYPES[dtype])
    x[1, cols // 2], x[2, cols - 1], x[3] = float("nan"), float("inf"), 0.0
    groups = -(-cols // 32)
    tiles = -(-groups // 4)
    for m in (sr.rms_norm(x, eps=0.0, format=fmt), sr.quantize(x, fmt)):
        scales = m.scales.view(tiles, 32, 4, 4)[:, :6, 0].permute(1, 0, 2).reshape(6, tiles * 4)
        assert (scales[:, groups:] == 0).all()
        data = m.data.view(6, -1)
        pad = data[:, (cols + 1) // 2:] if fmt == "mx4" else data[:, cols:]
        assert ((pad & (0x77 if fmt == "mx4" else 0x7F)) == 0).all()
        if fmt == "mx4" and cols % 2:
            assert ((data[:, cols // 2] >> 4 & 7) == 0).all()


def test_quantisation_of_more_than_2_30_rows():
    few = torch.randn(2, 8, generator=gen(99), device=DEV).bfloat16()
    want = sr.quantize(few[:1], "mx4")
    rows = 2 ** 30 + 3
    m = sr.quantize(few[:1].expand(rows, 8), "mx4")
    assert torch.equal(m.data[-1], want.data[0]) and torch.equal(m.data[::2 ** 20 + 7].unique(dim=0), want.data)
    last = (rows - 1) // 128 * 512 + (rows - 1) % 32 * 16 + (rows - 1) % 128 // 32 * 4
    assert torch.equal(m.scales[last:last + 4], want.scales[:4])


# ------------------------------------------------------------------------------------------ waits that run out
WAIT = r"""
#include "sr_ptx.cuh"
// A wait as the operators' kernels have it, on a barrier at which nothing arrives.
__global__ void wait_for_nothing(int* error)
{
    __shared__ uint64_t bar;
    __shared__ int gave_up;
    if (threadIdx.x == 0) {
        gave_up = 0;
        srx::mbar_init(srx::smem_u32(&bar), 1);
        srx::mbar_init_done();
    }
    __syncthreads();
    srx::mbar_wait_warp(srx::smem_u32(&bar), 0, &gave_up);
    __syncthreads();
    if (threadIdx.x == 0 && gave_up) atomicExch(error, 1);
}
extern "C" int run(int* error, void* stream)
{
    wait_for_nothing<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(error);
    return cudaGetLastError();
}
"""


def test_a_wait_that_runs_out_is_reported_to_everyone_until_it_is_reset(tmp_path):
    import ctypes
    import os
    import subprocess
    import threading
    from paper_1806_04965_b200 import build, operators
    source, lib = tmp_path / "wait.cu", tmp_path / "wait.so"
    source.write_text(WAIT)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-shared", *build.NVCC_FLAGS, "-I", build.CSRC, str(source), "-o", str(lib)])
    word = operators._library()._Z22sr_operator_error_wordv
    word.restype = ctypes.c_void_p
    sr.operator_status()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    wait = ctypes.CDLL(str(lib))
    assert wait.run(ctypes.c_void_p(word()), ctypes.c_void_p(a.cuda_stream)) == 0
    a.synchronize()
    seen = []

    def ask(stream):
        with torch.cuda.stream(stream):
            try:
                sr.operator_status()
                seen.append("ok")
            except sr.SrError as e:
                seen.append(e.status)
    try:
        ask(b)                                                  # another stream's owner first
        ask(a)
        t = threading.Thread(target=ask, args=(torch.cuda.Stream(),))
        t.start()
        t.join()
        assert seen == ["SR_ERR_TIMEOUT"] * 3
    finally:
        sr.operator_reset()
        torch.cuda.synchronize()
    for device in (None, 0, "cuda", "cuda:0", torch.device("cuda"), torch.device("cuda:0")):
        sr.operator_status(device)


def test_status_of_a_stream_that_is_captured_is_refused_and_the_capture_lives():
    x = torch.randn(4, 64, device=DEV)
    want = sr.rms_norm(x)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out = sr.rms_norm(x)
        with pytest.raises(sr.SrError):
            sr.operator_status()
    g.replay()
    assert torch.equal(out, want)
    sr.operator_status()


# ------------------------------------------------------------------------------------------ the head
def head_of(fmt, dtype, change=None, **kw):
    C, H, K, dk, dv, O = 70, 4, 2, 32, 48, 7
    r = np.random.RandomState(3)
    w = {"qkv": r.randn(H * dk + K * (dk + dv), C) / C ** 0.5, "o": r.randn(C, H * dv) / (H * dv) ** 0.5, "out": r.randn(O, C), "bias": r.randn(O),
         "norm_x": 1 + 0.3 * r.randn(C), "norm_o": 1 + 0.3 * r.randn(H * dv), "norm_h": 1 + 0.3 * r.randn(C), "log_decay": -np.array([0.05, 0.3])}
    if change:
        w[change] = w[change] * (1 + 0.5 * (np.arange(w[change].size).reshape(w[change].shape) % 2 == 0))
    return sr.TemporalHead(w, C, H, K, dk, dv, batch=3, format=fmt, dtype=dtype, **kw), w, (C, H, K, dk, dv, O)


@pytest.mark.parametrize("T", [1, 40, 150])
@pytest.mark.parametrize("fmt, dtype", [("mx4", "bf16"), ("mx8", "fp32"), ("mx4", "fp32"), ("mx8", "bf16")])
def test_head_is_the_public_calls_in_a_row(fmt, dtype, T):
    head, w, (C, H, K, dk, dv, O) = head_of(fmt, dtype, eps=1e-5)
    B, dt = 3, TYPES[dtype]
    w = {n: torch.tensor(x, dtype=torch.float32, device=DEV) for n, x in w.items()}
    wq = {n: sr.quantize(w[n], fmt) for n in ("qkv", "o", "out")}
    features = torch.randn(T, B, C, generator=gen(120), device=DEV)
    state = torch.zeros(B, K, dk, dv, device=DEV)

    def before(x):
        qkv = sr.product(sr.rms_norm(x, w["norm_x"], eps=1e-5, format=fmt), wq["qkv"], dtype=dt)
        return [t.reshape(len(x), -1, n) for t, n in zip(qkv.split((H * dk, K * dk, K * dv), dim=1), (dk, dk, dv))]

    def behind(x, o):
        y = sr.product(sr.rms_norm(o.reshape(len(x), H * dv), w["norm_o"], eps=1e-5, format=fmt), wq["o"], dtype=dt)
        return sr.product(sr.rms_norm(y, w["norm_h"], residual=x, eps=1e-5, format=fmt)[0], wq["out"], bias=w["bias"], dtype=torch.float32)
    x = features.view(T * B, C).to(dt)
    q, k, v = [t.view(T, B, *t.shape[1:]) for t in before(x)]
    o, last = sr.linear_attention_run(q, k, v, w["log_decay"], scale=dk ** -0.5)
    compare(q, k, v, w["log_decay"], None, o, last, dk ** -0.5, dtype, [(slice(None), b) for b in range(B)])
    assert torch.equal(head.run(features), behind(x, o).view(T, B, O)) and torch.equal(head.state, last)
    head.reset()
    for t in range(min(T, 20)):
        x = features[t].to(dt)
        o = sr.linear_attention_step(*before(x), w["log_decay"], state, scale=dk ** -0.5)
        assert torch.equal(head.step(features[t]), behind(x, o)) and torch.equal(head.state, state)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T, cuts", [(300, (128, 129)), (300, (1, 299)), (2000, (700, 1999))])
def test_clips_in_parts_and_frames_carry_the_whole_state_on(T, cuts, dtype):
    B, H, K, dk, dv = 2, 4, 2, 64, 48
    q, k, v, d = inputs((T, B), H, K, dk, dv, dtype, True, seed=121)
    d = d / 20
    state, outs, t0 = torch.zeros(B, K, dk, dv, device=DEV), [], 0
    for t1 in cuts + (T,):
        out, _ = sr.linear_attention_run(q[t0:t1], k[t0:t1], v[t0:t1], d[t0:t1], state=state, state_out=state, scale=0.2)
        outs.append(out)
        t0 = t1
    at = [(slice(None), b) for b in range(B)]
    compare(q, k, v, d, None, torch.cat(outs), state, 0.2, dtype, at)
    state.zero_()
    out, _ = sr.linear_attention_run(q[:T // 2], k[:T // 2], v[:T // 2], d[:T // 2], state=state, state_out=state, scale=0.2)
    outs = [out] + [sr.linear_attention_step(q[t], k[t], v[t], d[t], state, scale=0.2)[None] for t in range(T // 2, T)]
    compare(q, k, v, d, None, torch.cat(outs), state, 0.2, dtype, at)


@pytest.mark.parametrize("name", ["qkv", "o", "out", "bias", "norm_x", "norm_o", "norm_h", "log_decay"])
def test_every_weight_of_the_head_matters(name):
    features = torch.randn(30, 3, 70, generator=gen(122), device=DEV)
    a, b = head_of("mx8", "fp32")[0].run(features), head_of("mx8", "fp32", change=name)[0].run(features)
    # every second of its values is half as much again: outputs change by far more than what an element's rounding (2^-4) would move in one of 70 terms
    assert torch.linalg.vector_norm(a - b) > 0.02 * torch.linalg.vector_norm(a)
