"""The temporal head's operators on the GPU where their paths meet: precision, borders of segments and tiles, rows at the ends of the range.

Bounds as in test_gpu_operators.py; where they are tighter the test says why."""
import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from tests import operator_oracle as oracle
from tests.test_gpu_operators import DEV, TYPES, gen, host, inputs, within

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
