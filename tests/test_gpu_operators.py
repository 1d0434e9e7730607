"""The temporal head's operators on the GPU against their definitions in 64 bits (tests/operator_oracle.py).

Tolerances.  u is half a step of the output's type (bf16 2^-8, fp32 2^-24): the last rounding.  A sum of n terms in 32 bits is off by at most
n * 2^-23 times the sum of the terms' magnitudes (one unit in the last place of a partial sum for each addition; the tensor cores truncate), and
the factors of a term (decays: an exponential of a sum of up to T logarithms) by a few such steps each.  Where a kernel rounds a factor to bf16
ahead of a product of bf16 inputs (weights of the frames of a chunk, states), every term may be off by 2^-8 of its magnitude."""
import numpy as np
import pytest
import torch

import paper_1806_04965_b200 as sr
from paper_1806_04965_b200 import SrError
from tests import operator_oracle as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, want, bound):
    got = host(got)
    assert got.shape == want.shape
    assert (np.isnan(got) == np.isnan(want)).all()
    off = np.where(np.isnan(want), 0.0, np.abs(got - want))
    worst = float((off / np.maximum(bound, 1e-300)).max()) if off.size else 0.0
    assert worst <= 1.0, "%.3g times the bound" % worst


# ------------------------------------------------------------------------------------------ microscaled formats
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 32), (3, 31), (5, 33), (129, 128), (130, 200), (2, 4100), (7, 264), (1, 40000)])
def test_quantize_gives_the_layouts_codes(rows, cols, fmt, dtype):
    x = (torch.randn(rows, cols, generator=gen(1), device=DEV) * torch.exp(4 * torch.randn(rows, 1, generator=gen(2), device=DEV))).to(TYPES[dtype])
    m = sr.quantize(x, fmt)
    code, scales, values = oracle.quantize(host(x), fmt)
    data, placed = oracle.pack(code, scales, fmt)
    assert (m.data.cpu().numpy().ravel() == data.ravel()).all()
    got = m.scales.cpu().numpy()
    tg = -(-(-(-cols // 32)) // 4)
    for r in range(rows):                                       # rows that are there, padding groups among them
        at = (r // 128 * tg + np.arange(tg))[:, None] * 512 + r % 32 * 16 + r % 128 // 32 * 4 + np.arange(4)
        assert (got[at] == placed[at]).all()
    assert (host(m.values()) == values).all()


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
def test_quantize_at_its_borders(fmt):
    tops = {"mx4": 6.0, "mx8": 448.0}[fmt]
    rows = []
    for e in (-149, -130, -127, -126, -119, -60, 0, 1, 60, 118):
        for f in (1.0, 1.0 + 2.0 ** -23, 1.0 - 2.0 ** -24):
            rows.append([tops * f * 2.0 ** e] + [tops * 2.0 ** e * i / 61.0 * (-1) ** i for i in range(31)])
    table = oracle.E2M1 if fmt == "mx4" else oracle.E4M3
    mids = ((table[1:] + table[:-1]) / 2)
    for i in range(0, len(mids), 30):                           # ties, either sign
        rows.append([tops, -tops] + list(mids[i:i + 30]) + [0.0] * (30 - len(mids[i:i + 30])))
    rows.append([0.0] * 16 + [-0.0] * 16)
    rows.append([3.4028234e38, -1.0] + [1e38] * 30)
    x = torch.tensor(rows, dtype=torch.float64).float().to(DEV)
    m = sr.quantize(x, fmt)
    code, scales, values = oracle.quantize(host(x), fmt)
    assert (m.data.cpu().numpy().ravel() == oracle.pack(code, scales, fmt)[0].ravel()).all()
    assert (host(m.values()) == values.astype(np.float32)).all()


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
def test_a_group_that_is_not_finite_stands_for_nans_and_touches_its_row_only(fmt):
    x = torch.randn(140, 256, generator=gen(3), device=DEV)
    x[5, 40], x[131, 255], x[7, 0] = float("inf"), float("nan"), float("-inf")
    m = sr.quantize(x, fmt)
    values = host(m.values())
    bad = np.zeros((140, 256), bool)
    bad[5, 32:64] = bad[131, 224:256] = bad[7, 0:32] = True
    assert (np.isnan(values) == bad).all()
    y = host(sr.product(m, sr.quantize(torch.randn(70, 256, generator=gen(4), device=DEV), fmt), dtype=torch.float32))
    assert (np.isnan(y).all(1) == bad.any(1)).all() and (np.isnan(y).any(1) == bad.any(1)).all()


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows, cols, outs", [(1, 32, 1), (1, 1, 5), (3, 100, 17), (8, 4096, 128), (16, 1000, 1111), (33, 64, 130), (129, 129, 257), (300, 2048, 72),
                                              (513, 96, 600), (1000, 288, 40), (70, 5000, 300), (2100, 160, 1300), (1900, 1000, 2600), (1000, 4100, 2700), (577, 2048, 8300)])
def test_product(rows, cols, outs, fmt, dtype):
    a = torch.randn(rows, cols, generator=gen(5), device=DEV) * torch.exp(torch.randn(rows, cols, generator=gen(6), device=DEV))
    w = torch.randn(outs, cols, generator=gen(7), device=DEV)
    bias = torch.randn(outs, generator=gen(8), device=DEV)
    qa, qw = sr.quantize(a, fmt), sr.quantize(w, fmt)
    va, vw = host(qa.values()), host(qw.values())
    want, mag = va @ vw.T + host(bias), np.abs(va) @ np.abs(vw).T + np.abs(host(bias))
    bound = oracle.HALF_STEP[dtype] * np.abs(want) + (cols + 1) * 2.0 ** -23 * mag
    within(sr.product(qa, qw, bias=bias, dtype=TYPES[dtype]), want, bound)
    within(sr.product(qa, qw, bias=bias, relu=True, dtype=TYPES[dtype]), np.maximum(want, 0), bound)
    out = torch.full((rows, outs + 3), 7.0, dtype=TYPES[dtype], device=DEV)
    sr.product(qa, qw, out=out[:, :outs])                        # rows with gaps, no bias
    assert (out[:, outs:] == 7).all()
    within(out[:, :outs], want - host(bias), bound + oracle.HALF_STEP[dtype] * np.abs(host(bias)))
    again = sr.product(qa, qw, bias=bias, dtype=TYPES[dtype])
    assert torch.equal(again, sr.product(qa, qw, bias=bias, dtype=TYPES[dtype]))
    sr.operator_status()


def test_product_of_extreme_scales():
    # scales from 2^-127 to 2^120 in one matrix: a row's terms differ by less than 2^127 only where both operands say so
    a = torch.randn(64, 128, generator=gen(9), device=DEV) * torch.exp2(torch.linspace(-60, 60, 64, device=DEV))[:, None]
    w = torch.randn(48, 128, generator=gen(10), device=DEV) * torch.exp2(torch.linspace(-60, 60, 48, device=DEV))[:, None]
    for fmt in ("mx4", "mx8"):
        qa, qw = sr.quantize(a, fmt), sr.quantize(w, fmt)
        va, vw = host(qa.values()), host(qw.values())
        got, want, mag = sr.product(qa, qw, dtype=torch.float32), va @ vw.T, np.abs(va) @ np.abs(vw).T
        normal = mag > 2.0 ** -100
        assert normal.mean() > 0.7
        within(torch.where(torch.from_numpy(normal).to(DEV), got, torch.zeros_like(got)), np.where(normal, want, 0), 129 * 2.0 ** -23 * mag)


def test_product_without_rows_or_outputs():
    q = sr.quantize(torch.randn(4, 64, generator=gen(1), device=DEV))
    none = sr.quantize(torch.empty(0, 64, device=DEV))
    assert sr.product(none, q).shape == (0, 4) and sr.product(q, none).shape == (4, 0)


# ------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows, cols", [(1, 1), (5, 7), (3, 32), (9, 1003), (1, 1024), (130, 2048), (2, 4096), (3, 5000), (2, 33000), (1, 40001)])
def test_norm(rows, cols, residual, dtype):
    x = (3 * torch.randn(rows, cols, generator=gen(11), device=DEV)).to(TYPES[dtype])
    r = torch.randn(rows, cols, generator=gen(12), device=DEV).to(TYPES[dtype]) if residual else None
    w = torch.randn(cols, generator=gen(13), device=DEV)
    got = sr.rms_norm(x, w, residual=r, eps=1e-5)
    y, s = oracle.norm(host(x), host(w), None if r is None else host(r), 1e-5)
    # the sum in 32 bits (half a step), its square's sum (under the root: half of (cols + 3) steps), root, quotient and two products
    bound = (oracle.HALF_STEP[dtype] + ((cols + 3) / 2 + 8) * 2.0 ** -23) * np.abs(y)
    if residual:
        bound = bound + 2.0 ** -23 * np.abs(host(w)) * (np.abs(host(x)) + np.abs(host(r))) / np.sqrt((s * s).mean(-1, keepdims=True) + 1e-5)
        within(got[1], s, (oracle.HALF_STEP[dtype] + 2.0 ** -24) * np.abs(s))
        got = got[0]
    within(got, y, bound)
    plain = sr.rms_norm(x, eps=1e-5)
    within(plain, oracle.norm(host(x), eps=1e-5)[0], (oracle.HALF_STEP[dtype] + ((cols + 3) / 2 + 8) * 2.0 ** -23) * np.abs(oracle.norm(host(x), eps=1e-5)[0]))


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows, cols", [(1, 1), (4, 1024), (131, 200), (2, 5000), (3, 1003)])
def test_norm_with_microscaled_output(rows, cols, fmt, dtype):
    x = torch.randn(rows, cols, generator=gen(14), device=DEV).to(TYPES[dtype])
    r = torch.randn(rows, cols, generator=gen(15), device=DEV).to(TYPES[dtype])
    w = torch.rand(cols, generator=gen(16), device=DEV) + 0.5
    m, total = sr.rms_norm(x, w, residual=r, format=fmt)
    y, s = oracle.norm(host(x), host(w), host(r))
    values = host(m.values())
    # half a step of the element's type relative to the value, or to the smallest step of its group; a scale may be one higher where the
    # 32-bit result passes the border that the 64-bit one does not reach
    pad = np.zeros((rows, -(-cols // 32) * 32))
    pad[:, :cols] = np.abs(y)
    most = np.repeat(pad.reshape(rows, -1, 32).max(-1), 32, axis=1)[:, :cols] * (1 + 2.0 ** -10)
    step = most / 6 * 2 * 0.25 if fmt == "mx4" else most / 448 * 2 * 2.0 ** -10
    assert (np.abs(values - y) <= np.maximum(np.abs(y) * (0.25 if fmt == "mx4" else 2.0 ** -4), step) * (1 + 2.0 ** -10)).all()
    assert (host(total) == host((x.double() + r.double()).to(TYPES[dtype]))).all() if dtype == "bf16" else True
    # and exactly what quantising the fp32 norm of the same sums gives, where x is fp32
    if dtype == "fp32":
        again = sr.quantize(sr.rms_norm(x, w, residual=r)[0], fmt)
        assert torch.equal(m.data, again.data) and torch.equal(m.values(), again.values())


def test_norm_of_rows_with_gaps_zeros_and_nans():
    big = torch.randn(6, 200, generator=gen(17), device=DEV)
    x = big[:, 10:140]
    within(sr.rms_norm(x), oracle.norm(host(x))[0], 80 * 2.0 ** -23 * np.abs(oracle.norm(host(x))[0]))
    z = torch.zeros(3, 64, device=DEV)
    assert (sr.rms_norm(z) == 0).all()
    z[1, 3] = float("nan")
    assert torch.isnan(sr.rms_norm(z)[1]).all() and (sr.rms_norm(z)[0::2] == 0).all()


# ------------------------------------------------------------------------------------------ linear attention
def inputs(lead, heads, groups, dk, dv, dtype, gated, seed=20):
    g = gen(seed)
    q = torch.randn(*lead, heads, dk, generator=g, device=DEV).to(TYPES[dtype])
    k = (torch.randn(*lead, groups, dk, generator=g, device=DEV) / dk ** 0.5).to(TYPES[dtype])
    v = torch.randn(*lead, groups, dv, generator=g, device=DEV).to(TYPES[dtype])
    d = -torch.rand(*(lead if gated else ()), groups, generator=g, device=DEV) ** 3
    return q, k, v, d


def check_run(q, k, v, d, state, out, last, scale, dtype, sequences):
    """sequences: per sequence the index of its frames in the leading dimensions."""
    for b, at in enumerate(sequences):
        n = q[at].shape[0]
        dd = host(d if d.dim() == 1 else d[at])
        want, S, mag, A = oracle.attention(host(q[at]), host(k[at]), host(v[at]), dd, None if state is None else host(state[b]), scale)
        steps = (2 * n + q.shape[-1] + 40) * 2.0 ** -23
        extra = 2 * 2.0 ** -8 if dtype == "bf16" else 0.0
        within(out[at], want, oracle.HALF_STEP[dtype] * np.abs(want) + (steps + extra) * mag)
        within(last[b], S, steps * A)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T, B, heads, groups, dk, dv", [(1, 1, 1, 1, 1, 1), (2, 3, 4, 2, 64, 64), (63, 2, 2, 2, 64, 64), (64, 1, 2, 1, 128, 128),
                                                         (65, 2, 1, 1, 64, 128), (127, 1, 2, 2, 128, 64), (128, 2, 8, 2, 32, 48), (129, 3, 3, 3, 40, 72), (300, 2, 4, 4, 25, 33),
                                                         (257, 1, 2, 2, 128, 128), (700, 1, 3, 1, 64, 64), (40, 2, 1, 1, 256, 16), (513, 1, 1, 1, 96, 200), (20, 1, 40, 1, 16, 8)])
def test_run(T, B, heads, groups, dk, dv, gated, dtype):
    q, k, v, d = inputs((T, B), heads, groups, dk, dv, dtype, gated)
    state = torch.randn(B, groups, dk, dv, generator=gen(21), device=DEV)
    at = [(slice(None), b) for b in range(B)]
    out, last = sr.linear_attention_run(q, k, v, d, state=state, scale=0.3)
    check_run(q, k, v, d, state, out, last, 0.3, dtype, at)
    out, last = sr.linear_attention_run(q, k, v, d)
    check_run(q, k, v, d, None, out, last, 1.0, dtype, at)
    again, last2 = sr.linear_attention_run(q, k, v, d)
    assert torch.equal(out, again) and torch.equal(last, last2)
    kept = state.clone()
    out2, same = sr.linear_attention_run(q, k, v, d, state=kept, scale=0.3, state_out=kept)
    out, last = sr.linear_attention_run(q, k, v, d, state=state, scale=0.3)
    assert same is kept and torch.equal(kept, last) and torch.equal(out2, out)
    sr.operator_status()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T, B, heads, groups, dk, dv", [(9, 80, 4, 4, 25, 30), (15, 60, 4, 4, 64, 64), (33, 50, 6, 3, 128, 72), (7, 100, 2, 2, 200, 20)])
def test_run_of_many_sequences(T, B, heads, groups, dk, dv, dtype):
    q, k, v, d = inputs((T, B), heads, groups, dk, dv, dtype, True)
    state = torch.randn(B, groups, dk, dv, generator=gen(28), device=DEV)
    out, last = sr.linear_attention_run(q, k, v, d, state=state, scale=0.3)
    check_run(q, k, v, d, state, out, last, 0.3, dtype, [(slice(None), b) for b in range(B)])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lengths, heads, groups, dk, dv", [([0, 1, 130, 0, 64, 700, 3], 4, 2, 64, 64), ([5], 1, 1, 128, 128), ([0, 0], 2, 2, 64, 64), ([1] * 9, 2, 1, 40, 24),
                                                            ([900, 2, 0, 129], 2, 2, 128, 128)])
def test_run_of_packed_sequences(lengths, heads, groups, dk, dv, dtype):
    spare = 17                                                  # frames behind the last sequence
    total = sum(lengths) + spare
    q, k, v, d = inputs((total,), heads, groups, dk, dv, dtype, True)
    for t in (q, k, v):
        t[sum(lengths):] = float("nan")
    first = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    offsets = torch.tensor(first, dtype=torch.int64, device=DEV)
    state = torch.randn(len(lengths), groups, dk, dv, generator=gen(22), device=DEV)
    out = torch.full((total, heads, dv), 5.0, dtype=TYPES[dtype], device=DEV)
    _, last = sr.linear_attention_run(q, k, v, d, state=state, offsets=offsets, scale=0.5, out=out)
    check_run(q, k, v, d, state, out, last, 0.5, dtype, [slice(a, b) for a, b in zip(first, first[1:])])
    assert (out[sum(lengths):] == 5).all()
    for b, n in enumerate(lengths):
        if n == 0:
            assert torch.equal(last[b], state[b])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T, B, heads, dk, dv", [(5000, 1, 1, 64, 64), (3001, 2, 1, 128, 128), (4097, 1, 2, 40, 72)])
def test_long_runs(T, B, heads, dk, dv, dtype):
    q, k, v, d = inputs((T, B), heads, heads, dk, dv, dtype, True)
    d = d / 20
    state = torch.randn(B, heads, dk, dv, generator=gen(23), device=DEV)
    out, last = sr.linear_attention_run(q, k, v, d, state=state)
    check_run(q, k, v, d, state, out, last, 1.0, dtype, [(slice(None), b) for b in range(B)])
    a, mid = sr.linear_attention_run(q[:1234], k[:1234], v[:1234], d[:1234], state=state)        # in two parts
    b, end = sr.linear_attention_run(q[1234:], k[1234:], v[1234:], d[1234:], state=mid)
    check_run(q, k, v, d, state, torch.cat((a, b)), end, 1.0, dtype, [(slice(None), b) for b in range(B)])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dk, dv", [(64, 64), (128, 128), (40, 72)])
def test_decays_at_their_borders(dk, dv, dtype):
    # no decay at all, decay to nothing within a frame, a state that starts anew in the middle of a chunk and at its border
    T = 200
    q, k, v, d = inputs((T, 1), 3, 3, dk, dv, dtype, True)
    d[:, :, 0] = 0.0
    d[:, :, 1] = -200.0
    d[37, :, 2] = d[64, :, 2] = d[128, :, 2] = d[129, :, 2] = float("-inf")
    d[100:110, :, 2] = -1e30
    state = torch.randn(1, 3, dk, dv, generator=gen(24), device=DEV)
    out, last = sr.linear_attention_run(q, k, v, d, state=state)
    check_run(q, k, v, d, state, out, last, 1.0, dtype, [(slice(None), 0)])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_run_of_views(dtype):
    # queries, keys and values side by side in the rows of one product, decays shared by all sequences, an odd offset
    T, B, H, G, dk, dv = 70, 3, 4, 2, 64, 64
    n = H * dk + G * (dk + dv)
    for lead in (0, 1, 8):
        big = torch.randn(T * B, n + lead, generator=gen(25), device=DEV).to(TYPES[dtype])[:, lead:]
        q = big[:, :H * dk].unflatten(0, (T, B)).unflatten(2, (H, dk))
        k = big[:, H * dk:H * dk + G * dk].unflatten(0, (T, B)).unflatten(2, (G, dk))
        v = big[:, H * dk + G * dk:].unflatten(0, (T, B)).unflatten(2, (G, dv))
        d = -torch.rand(T, 1, G, generator=gen(26), device=DEV).expand(T, B, G)
        out, last = sr.linear_attention_run(q, k, v, d, scale=0.1)
        check_run(q, k, v, d, None, out, last, 0.1, dtype, [(slice(None), b) for b in range(B)])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B, heads, groups, dk, dv", [(1, 1, 1, 1, 1), (1, 8, 8, 64, 64), (3, 4, 2, 128, 128), (2, 6, 6, 40, 72), (5, 12, 1, 25, 33), (2, 2, 2, 256, 16),
                                                      (1, 128, 1, 64, 40), (37, 3, 3, 128, 64)])
def test_step(B, heads, groups, dk, dv, dtype):
    state = torch.randn(B, groups, dk, dv, generator=gen(27), device=DEV)
    for gated in (False, True):
        q, k, v, d = inputs((B,), heads, groups, dk, dv, dtype, gated)
        was = state.clone()
        out = sr.linear_attention_step(q, k, v, d, state, scale=0.7)
        for b in range(B):
            want, S, mag, A = oracle.attention(host(q[b:b + 1]), host(k[b:b + 1]), host(v[b:b + 1]), host(d if not gated else d[b:b + 1]), host(was[b]), 0.7)
            within(out[b:b + 1], want, oracle.HALF_STEP[dtype] * np.abs(want) + (dk + 20) * 2.0 ** -23 * mag)
            within(state[b], S, 8 * 2.0 ** -23 * A)


def test_runs_without_frames_or_sequences():
    for dtype in ("bf16", "fp32"):
        q, k, v, d = inputs((0, 3), 2, 2, 64, 64, dtype, True)
        state = torch.randn(3, 2, 64, 64, generator=gen(28), device=DEV)
        out, last = sr.linear_attention_run(q, k, v, d, state=state)
        assert out.shape == (0, 3, 2, 64) and torch.equal(last, state)
        assert (sr.linear_attention_run(q, k, v, d)[1] == 0).all()
        out, last = sr.linear_attention_run(q[:, 0], k[:, 0], v[:, 0], d[:, 0], offsets=torch.zeros(4, dtype=torch.int64, device=DEV), state=state)
        assert torch.equal(last, state)
        q, k, v, d = inputs((40,), 2, 2, 64, 64, dtype, True)
        out, last = sr.linear_attention_run(q, k, v, d, offsets=torch.zeros(1, dtype=torch.int64, device=DEV), out=torch.full((40, 2, 64), 3.0, dtype=TYPES[dtype], device=DEV))
        assert last.shape == (0, 2, 64, 64) and (out == 3).all()
        assert sr.linear_attention_step(q[:0], k[:0], v[:0], d[:0], last).shape == (0, 2, 64)


def test_steps_are_a_run():
    T, B, H, dk, dv = 150, 2, 2, 64, 64
    q, k, v, d = inputs((T, B), H, H, dk, dv, "fp32", True)
    state = torch.zeros(B, H, dk, dv, device=DEV)
    out = torch.stack([sr.linear_attention_step(q[t], k[t], v[t], d[t], state) for t in range(T)])
    check_run(q, k, v, d, None, out, state, 1.0, "fp32", [(slice(None), b) for b in range(B)])
    want, last = sr.linear_attention_run(q, k, v, d)
    check_run(q, k, v, d, None, want, last, 1.0, "fp32", [(slice(None), b) for b in range(B)])


def test_values_that_are_not_finite_stay_in_their_sequence_and_head():
    T, B, H, D = 140, 2, 2, 64
    for dtype in ("bf16", "fp32"):
        q, k, v, d = inputs((T, B), H, H, D, D, dtype, False)
        clean, last = sr.linear_attention_run(q, k, v, d)
        v[70, 0, 1, 5] = float("nan")
        out, end = sr.linear_attention_run(q, k, v, d)
        assert torch.equal(out[:, 1], clean[:, 1]) and torch.equal(out[:, 0, 0], clean[:, 0, 0]) and torch.equal(end[1], last[1])
        assert torch.equal(out[:70, 0, 1], clean[:70, 0, 1])              # frames before it do not see it
        assert torch.isnan(out[70:, 0, 1, 5]).all() and torch.isnan(end[0, 1, :, 5]).all()
        keep = [c for c in range(D) if c != 5]
        assert torch.equal(out[:, 0, 1][:, keep], clean[:, 0, 1][:, keep])


# ------------------------------------------------------------------------------------------ places beyond 2^31 elements, inputs repeated by strides
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_frames_that_lie_far_apart(dtype):
    T, B, H, D, gap = 300, 2, 2, 64, 7_500_000
    q, k, v, d = inputs((T, B), H, H, D, D, dtype, True)
    room = torch.empty(T * gap, dtype=TYPES[dtype], device=DEV)
    far = []
    for i, x in enumerate((q, k, v)):
        far.append(room[i * 4096:].as_strided((T, B, H, D), (gap, H * D, D, 1)))
        far[i].copy_(x)
    out, last = sr.linear_attention_run(*far, d, scale=0.2)
    check_run(q, k, v, d, None, out, last, 0.2, dtype, [(slice(None), b) for b in range(B)])


def test_states_of_more_than_2_31_elements():
    B, G, D, T = 2 ** 31 // (16 * 128 * 128) + 1, 16, 128, 16
    state = torch.zeros(B, G, D, D, device=DEV)
    state[-1].normal_(generator=gen(40))
    was = state[-1:].clone()
    q, k, v, d = inputs((B,), G, G, D, D, "bf16", False)
    out = sr.linear_attention_step(q, k, v, d, state, scale=0.5)
    want, S, mag, A = oracle.attention(host(q[-1:]), host(k[-1:]), host(v[-1:]), host(d), host(was[0]), 0.5)
    within(out[-1:], want, 2.0 ** -8 * np.abs(want) + (D + 20) * 2.0 ** -23 * mag)
    within(state[-1], S, 8 * 2.0 ** -23 * A)
    was = state[-2:].clone()
    q, k, v, d = inputs((T, B), G, G, D, D, "bf16", False)
    out, _ = sr.linear_attention_run(q, k, v, d, state=state, scale=0.5, state_out=state)
    check_run(q[:, -2:], k[:, -2:], v[:, -2:], d, was, out[:, -2:], state[-2:], 0.5, "bf16", [(slice(None), 0), (slice(None), 1)])


def test_rows_beyond_2_31_elements():
    rows, cols = 2 ** 16 + 131, 2 ** 15
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV).normal_(generator=gen(41))
    w = torch.randn(cols, generator=gen(42), device=DEV)
    out, total = sr.rms_norm(x, w, residual=x, eps=1e-5)
    want, s = oracle.norm(host(x[-3:]), host(w), host(x[-3:]), 1e-5)
    assert torch.equal(total[-3:], x[-3:] * 2)
    within(out[-3:], want, (2.0 ** -8 + ((cols + 3) / 2 + 8) * 2.0 ** -23) * np.abs(want))        # (the sums of equal rows are exact)
    del out, total
    m = sr.quantize(x, "mx4")
    few = sr.quantize(x[-131:].contiguous(), "mx4")              # (the first row of a tile of scales)
    assert torch.equal(m.data[-131:], few.data)
    full = (rows // 128 - 1) * (cols // 128) * 512               # the last two tiles of rows: 128 and 3 of them
    a, b = m.scales[full:].view(2, -1, 32, 4, 4), few.scales.view(2, -1, 32, 4, 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1, :, :3, 0], b[1, :, :3, 0])
    del m, few
    narrow, wide = sr.quantize(x[:, :64], "mx8"), sr.quantize(x[:2 ** 15, :64], "mx8")
    y = sr.product(narrow, wide)
    va, vw = host(narrow.values()[-3:]), host(wide.values())
    within(y[-3:], va @ vw.T, 2.0 ** -8 * np.abs(va @ vw.T) + 65 * 2.0 ** -23 * (np.abs(va) @ np.abs(vw).T))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_inputs_that_strides_repeat(dtype):
    T, B, H, D = 140, 3, 4, 64
    q, k, v, d = inputs((T, 1), H, H, D, D, dtype, True)
    q = torch.randn(T, B, H, D, generator=gen(43), device=DEV).to(TYPES[dtype])
    k, v, d = k.expand(T, B, H, D), v[:, :, :1].expand(T, B, H, D), d.expand(T, B, H)
    out, last = sr.linear_attention_run(q, k, v, d, scale=0.2)
    check_run(q, k, v, d, None, out, last, 0.2, dtype, [(slice(None), b) for b in range(B)])
    state = torch.zeros(B, H, D, D, device=DEV)
    one = sr.linear_attention_step(q[0], k[0], v[0], d[0], state, scale=0.2)
    for b in range(B):
        want, S, mag, A = oracle.attention(host(q[:1, b]), host(k[:1, b]), host(v[:1, b]), host(d[:1, b]), None, 0.2)
        within(one[b:b + 1], want, oracle.HALF_STEP[dtype] * np.abs(want) + (D + 20) * 2.0 ** -23 * mag)
        within(state[b], S, 8 * 2.0 ** -23 * A)


def test_threads_call_at_the_same_time_on_their_own_streams():
    import threading
    cases = []
    for i in range(4):
        q, k, v, d = inputs((3000, 1), 2, 2, 64, 64, "bf16" if i % 2 else "fp32", True, seed=50 + i)     # (cut: with a workspace)
        x = torch.randn(30 + i, 512, generator=gen(60 + i), device=DEV).bfloat16()
        cases.append((q, k, v, d, x, sr.quantize(torch.randn(200, 512, generator=gen(70 + i), device=DEV))))

    def calls(c):
        out, last = sr.linear_attention_run(*c[:4])
        return out, last, sr.linear_attention_step(c[0][0], c[1][0], c[2][0], c[3][0], last), sr.product(sr.rms_norm(c[4], format="mx4"), c[5])
    want = [calls(c) for c in cases]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = calls(cases[i])
                torch.cuda.current_stream().synchronize()
                bad.extend((i, n) for n, (a, b) in enumerate(zip(got, want[i])) if not torch.equal(a, b))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


# ------------------------------------------------------------------------------------------ streams, graphs, refusals, the head
def test_calls_are_captured_and_replayed_on_another_stream():
    T, B, H, D = 200, 2, 2, 64
    q, k, v, d = inputs((T, B), H, H, D, D, "bf16", True)
    x = torch.randn(40, 256, generator=gen(30), device=DEV).bfloat16()
    w = sr.quantize(torch.randn(96, 256, generator=gen(31), device=DEV))

    def calls():
        out, last = sr.linear_attention_run(q, k, v, d)
        one = sr.linear_attention_step(q[0], k[0], v[0], d[0], last)
        return out, last, one, sr.product(sr.rms_norm(x, format="mx4"), w)
    want = calls()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        calls()
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                got = calls()
            graphs.append((g, got))
    x2, q2 = x.clone(), q.clone()
    x.mul_(2), q.mul_(-1)
    other = calls()
    x.copy_(x2), q.copy_(q2)
    torch.cuda.synchronize()
    for g, got in graphs + graphs:
        with torch.cuda.stream(stream):
            g.replay()
        stream.synchronize()
        for a, b, c in zip(got, want, other):
            assert torch.equal(a, b)
        assert not torch.equal(got[0], other[0])


def test_large_products_and_runs_side_by_side_on_streams():
    # tiles of pairs of CTAs and chunks, which want whole SMs, and what is captured of them replayed beside the calls themselves
    cases = []
    for i, (rows, cols, outs, fmt) in enumerate([(1000, 4100, 2700, "mx4"), (1900, 1000, 2600, "mx8")]):
        x, w = torch.randn(rows, cols, generator=gen(80 + i), device=DEV), torch.randn(outs, cols, generator=gen(82 + i), device=DEV)
        cases.append((sr.quantize(x, fmt), sr.quantize(w, fmt)))
    q, k, v, d = inputs((300, 40), 4, 4, 64, 64, "bf16", True, seed=84)
    calls = [lambda: sr.product(*cases[0]), lambda: sr.product(*cases[1]), lambda: sr.linear_attention_run(q, k, v, d)[0]]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    graphs = []
    for c, s in zip(calls, streams):
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                graphs.append([g, c()])
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for c, s, (g, _) in zip(calls, streams, graphs):
            with torch.cuda.stream(s):
                got.append(c())
                g.replay()
        torch.cuda.synchronize()
        for a, (_, b), e in zip(got, graphs, want):
            assert torch.equal(a, e) and torch.equal(b, e)
    sr.operator_status()


def test_infinite_values_give_what_the_formula_gives():
    # +inf in the values: earlier frames do not see it, later ones are infinite with the weights' signs or NaN where those meet
    T, D = 150, 64
    for dtype in ("bf16", "fp32"):
        q, k, v, d = inputs((T, 1), 1, 1, D, D, dtype, False)
        q, k = q.abs(), k.abs()
        clean, _ = sr.linear_attention_run(q, k, v, d)
        v[40, 0, 0, 3], v[140, 0, 0, 9] = float("inf"), float("-inf")
        out, last = sr.linear_attention_run(q, k, v, d)
        assert torch.equal(out[:40], clean[:40])
        assert (out[40:, 0, 0, 3] == float("inf")).all() and (out[140:, 0, 0, 9] == float("-inf")).all() and torch.equal(out[:140, 0, 0, 9], clean[:140, 0, 0, 9])
        assert (last[0, 0, :, 3] == float("inf")).all() and (last[0, 0, :, 9] == float("-inf")).all()


def test_first_calls_of_a_process_may_be_captured():
    import subprocess
    import sys
    code = """
import torch
import paper_1806_04965_b200 as sr
q = torch.randn(200, 2, 2, 64, device="cuda:0").bfloat16()
d = -torch.rand(2, device="cuda:0")
x = torch.randn(20, 256, device="cuda:0").bfloat16()
g = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g):
    out, last = sr.linear_attention_run(q, q, q, d)
    one = sr.linear_attention_step(q[0], q[0], q[0], d, last)
    m = sr.rms_norm(x, format="mx4")
    y = sr.product(m, sr.quantize(x))
g.replay()
torch.cuda.synchronize()
want = sr.linear_attention_run(q, q, q, d)
assert torch.equal(out, want[0])
assert torch.equal(y, sr.product(sr.rms_norm(x, format="mx4"), sr.quantize(x)))
print("ok")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stderr[-1500:]


def test_calls_without_the_compiled_marshalling_give_the_same(monkeypatch):
    q, k, v, d = inputs((70, 2), 4, 2, 64, 48, "bf16", True)
    x, w = torch.randn(9, 200, generator=gen(33), device=DEV), torch.rand(200, generator=gen(34), device=DEV)

    def calls():
        state = torch.ones(2, 2, 64, 48, device=DEV)
        out, last = sr.linear_attention_run(q, k, v, d, state=state, scale=0.3)
        flat = [t.flatten(0, 1) for t in (q, k, v, d)]
        packed = sr.linear_attention_run(*flat, offsets=torch.tensor([0, 30, 140], device=DEV), state=state, out=torch.zeros(140, 4, 48, dtype=torch.bfloat16, device=DEV))
        one = sr.linear_attention_step(q[0], k[0], v[0], d[0], last)
        m, total = sr.rms_norm(x, w, residual=x, format="mx8")
        n = sr.quantize(x, "mx8")
        return [out, last, one, *packed, m.values(), total, sr.rms_norm(x), n.values(), sr.product(m, n, bias=w[:9].contiguous(), relu=True, dtype=torch.float32),
                sr.product(m, n, out=torch.zeros(9, 12, dtype=torch.bfloat16, device=DEV)[:, :9])]
    want = calls()
    for name in ("quantize", "product", "rms_norm", "run", "step"):
        monkeypatch.setattr(sr.operators._compiled, name, lambda *_: None)
    for a, b in zip(calls(), want):
        assert torch.equal(a, b)


def test_refusals():
    q, k, v, d = inputs((4, 2), 4, 2, 64, 64, "bf16", True)
    state = torch.zeros(2, 2, 64, 64, device=DEV)
    for bad in (lambda: sr.linear_attention_run(q, k.float(), v, d), lambda: sr.linear_attention_run(q, k, v, d.double()), lambda: sr.linear_attention_run(q[:, :, :3], k, v, d),
                lambda: sr.linear_attention_run(q, k[:3], v, d), lambda: sr.linear_attention_run(q, k, v, d[:, :1]), lambda: sr.linear_attention_run(q, k, v, d, state=state[:1]),
                lambda: sr.linear_attention_run(q, k, v, d, state=state.transpose(2, 3)), lambda: sr.linear_attention_run(q.transpose(2, 3), k, v, d),
                lambda: sr.linear_attention_run(q[:, 0], k[:, 0], v[:, 0], d[:, 0], offsets=torch.zeros(3, dtype=torch.int32, device=DEV)),
                lambda: sr.linear_attention_run(q, k, v, d, offsets=torch.zeros(3, dtype=torch.int64, device=DEV)), lambda: sr.linear_attention_run(q, k, v, d.cpu()),
                lambda: sr.linear_attention_step(q, k, v, d, state), lambda: sr.linear_attention_step(q[0], k[0], v[0], d[0], state.bfloat16()),
                lambda: sr.linear_attention_run(q.clone().requires_grad_(), k, v, d), lambda: sr.quantize(q[0, 0].t()), lambda: sr.quantize(q[0, 0].half()), lambda: sr.quantize(q[0, 0], "mx6"),
                lambda: sr.rms_norm(q[0, 0], torch.ones(63, device=DEV)), lambda: sr.rms_norm(q[0, 0], residual=q[0, 0].float()),
                lambda: sr.product(sr.quantize(q[0, 0]), sr.quantize(q[0, 0], "mx8")), lambda: sr.product(sr.quantize(q[0, 0]), sr.quantize(q[0, 0]), bias=torch.ones(3, device=DEV)),
                lambda: sr.product(sr.quantize(q[0, 0]), sr.quantize(q[0, 0]), dtype=torch.float16), lambda: sr.linear_attention_run(k, k, v, d, out=v)):
        with pytest.raises(SrError):
            bad()
    assert torch.isfinite(sr.linear_attention_run(q, k, v, d)[0].float()).all()


def test_offsets_that_are_out_of_range_reach_nothing_beyond_the_frames():
    q, k, v, d = inputs((50,), 2, 2, 64, 64, "bf16", True)
    out = torch.zeros(50, 2, 64, dtype=torch.bfloat16, device=DEV)
    offsets = torch.tensor([-5, 20, 10, 1 << 40], dtype=torch.int64, device=DEV)          # 0..20, empty, 10..50
    _, last = sr.linear_attention_run(q, k, v, d, offsets=offsets, out=out)
    assert (last[1] == 0).all() and torch.isfinite(last).all() and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("fmt, dtype", [("mx4", "bf16"), ("mx8", "fp32")])
def test_head_behind_a_rollout(fmt, dtype):
    """norm, product, attention, product and the residual's norm together, behind a network's rollout; clips, frames and windows of clips agree."""
    from tests.parity import make_graph, to_device
    from workloads import data, graphs
    spec = graphs.build("c2", batch=4, frames=12)
    G = make_graph(spec, "streaming", weights=data.make_weights(spec), biases=data.make_biases(spec))
    frames = [to_device(spec, data.make_inputs(spec)[v]) for v in G.input_nodes]
    C, H, K, dk, dv, O = 10, 4, 2, 32, 48, 7
    r = np.random.RandomState(3)
    w = {"qkv": r.randn(H * dk + K * (dk + dv), C) / C ** 0.5, "o": r.randn(C, H * dv) / (H * dv) ** 0.5, "out": r.randn(O, C), "bias": r.randn(O),
         "norm_x": 1 + 0.1 * r.randn(C), "norm_o": 1 + 0.1 * r.randn(H * dv), "norm_h": 1 + 0.1 * r.randn(C), "log_decay": -np.array([0.05, 0.3])}
    head = sr.TemporalHead(w, C, H, K, dk, dv, batch=4, format=fmt, dtype=dtype)
    features = G.rollout(frames)
    got = G.rollout(frames, head=head)
    end = head.get_state()
    assert got.shape == (12, 4, O) and torch.isfinite(got).all()
    # the plain head in 64 bits with the same roundings to the microscaled format
    def q(x):
        return oracle.quantize(x, fmt)[2]
    wq = {n: q(w[n].astype(np.float32)) for n in ("qkv", "o", "out")}
    x = host(features).reshape(48, C)
    n = H * dk, (H + K) * dk
    qkv = q(oracle.norm(x, w["norm_x"])[0]) @ wq["qkv"].T
    o = np.zeros((12, 4, H, dv))
    for b in range(4):
        part = qkv.reshape(12, 4, -1)[:, b]
        o[:, b] = oracle.attention(part[:, :n[0]].reshape(12, H, dk), part[:, n[0]:n[1]].reshape(12, K, dk), part[:, n[1]:].reshape(12, K, dv), w["log_decay"], scale=dk ** -0.5)[0]
    h = x + q(oracle.norm(o.reshape(48, -1), w["norm_o"])[0]) @ wq["o"].T
    want = (q(oracle.norm(h, w["norm_h"])[0]) @ wq["out"].T + w["bias"]).reshape(12, 4, O)
    # three roundings to the format lie between: a value next to a border may fall to its other side, so the outputs as a whole are compared.  Each of the three
    # rounds its element by up to half a step (mx4 1/4, mx8 2^-4) where that happens; that all of them do bounds the difference
    assert np.linalg.norm(host(got) - want) <= 3 * (0.25 if fmt == "mx4" else 2.0 ** -4) * np.linalg.norm(want)
    head.reset()
    steps = torch.stack([head.step(features[t]) for t in range(12)])
    near = 3 * (0.25 if fmt == "mx4" else 2.0 ** -4)
    assert torch.linalg.vector_norm(steps - got) <= near * torch.linalg.vector_norm(got)
    assert torch.linalg.vector_norm(head.state - end) <= near * torch.linalg.vector_norm(end)
    head.reset()
    parts = torch.cat((head.run(features[:5]), head.run(features[5:])))
    assert torch.linalg.vector_norm(parts - got) <= near * torch.linalg.vector_norm(got)
    head.set_state(end)
    assert torch.equal(head.get_state(), end)
    assert torch.equal(G.rollout(frames, head=head), got)
