"""Operators of the temporal head that stands behind a rollout: what they cost, and what they have to compute.

The head reads the features that a network gives for every frame.  Its parts: a root-mean-square norm with the residual's
addition, products with weights held in microscaled 4- or 8-bit floating point, and linear attention with a decay for each
head over the frames, for whole clips ("run") or frame by frame ("step").

Microscaled format.  A matrix [rows][cols] is cut along its columns into groups of 32.  A group has one scale 2^k, the
smallest power of two (not below 2^-127) with max|x| <= M * 2^k, M = 6 for "mx4" (e2m1) and 448 for "mx8" (e4m3), held as
the byte k + 127; its elements are x / 2^k, rounded to nearest even.  data: [rows][padded cols / 2] (mx4: element 2i in
the low half of byte i) or [rows][padded cols] (mx8), columns padded with zeros to a multiple of 32.  scales: the byte of row r,
group g lies in tile (r / 128, g / 4), tiles of 512 bytes row by row, at (r % 32) * 16 + (r % 128 / 32) * 4 + g % 4.

Keys of a case:
  op       "run", "step" (linear attention), "norm", "product" (quantisation of the rows, product with weights), or
           "norm_product" (norm with quantised output, product)
  dtype    type of the inputs and outputs: "bf16" or "fp32"
  run, step:  batch sequences, frames each (run), heads (of queries), groups (heads of keys, values and states), dk, dv;
           packed: sequences of different lengths one behind the other instead of [frames][batch]; gated: a decay for each
           frame and head instead of one for each head
  norm:    rows, cols; residual: whether something is added first
  product: rows, cols (of the activations), outs (rows of the weights), format "mx4" or "mx8", relu
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5


def _attend(name, op, batch, frames, heads, groups, dk, dv, dtype="bf16", packed=False, gated=False):
    return {"name": name, "op": op, "batch": batch, "frames": frames, "heads": heads, "groups": groups, "dk": dk, "dv": dv, "dtype": dtype,
            "packed": packed, "gated": gated}


def _norm(name, rows, cols, dtype, residual):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual}


def _product(name, op, rows, cols, outs, format, dtype="bf16", relu=False):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "outs": outs, "format": format, "dtype": dtype, "relu": relu}


def listed():
    return [
        # a batch of clips, frames-major as a rollout gives them: 32 sequences of 128 frames
        _attend("run_clips_b32", "run", 32, 128, 8, 8, 64, 64),
        # sequences of different lengths one behind the other, an empty one and one of a single frame among them, queries that share keys and values
        _attend("run_packed_b16", "run", 16, 3000, 16, 4, 128, 128, packed=True, gated=True),
        # one very long sequence, few heads: nothing to spread over the SMs but the sequence itself
        _attend("run_long_b1", "run", 1, 32768, 8, 8, 128, 128, gated=True),
        # validation in fp32, odd head sizes
        _attend("run_fp32_odd", "run", 5, 500, 6, 6, 40, 72, dtype="fp32"),
        # live, one sequence, one frame per call: all latency
        _attend("step_b1", "step", 1, 1, 8, 8, 64, 64),
        # many live sequences: the states are read and written once per frame
        _attend("step_b256", "step", 256, 1, 16, 16, 128, 128, gated=True),
        # features of a few live sequences
        _norm("norm_b8", 8, 1024, "bf16", True),
        # features of a batch of clips (128 frames x 128 sequences) in fp32, an odd width
        _norm("norm_clips_fp32", 16384, 1003, "fp32", True),
        # one live sequence: the weights are read once per frame
        _product("product_mx4_b1", "product", 1, 4096, 4096, "mx4", relu=True),
        # all frames of a batch of clips at once: the largest work
        _product("product_mx4_8192", "product", 8192, 4096, 8192, "mx4"),
        # 8 bits, fp32 features, odd sizes throughout
        _product("product_mx8_fp32_odd", "product", 777, 1000, 1111, "mx8", dtype="fp32", relu=True),
        # the head's first half on a batch of clips: norm with 8-bit output, product to queries, keys and values
        _product("norm_product_mx8", "norm_product", 4096, 1024, 4608, "mx8"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["run", "run", "run", "step", "step", "norm", "product", "product", "product", "norm_product"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op in ("run", "step"):
        groups = rng.choice([1, 2, 4, 6, 8, 16])
        heads = groups * rng.choice([1, 1, 1, 2, 4])
        dk, dv = rng.choice([(64, 64), (64, 64), (128, 128), (128, 128), (64, 128), (128, 64), (32, 48), (40, 72), (96, 80), (25, 33), (16, 128)])
        batch = _log_int(rng, 1, 256 if op == "step" else 64)
        frames = 1
        if op == "run":
            frames = max(2, min(_log_int(rng, 2, 16384), (1 << 22) // (batch * heads * max(dk, dv) // 8)))
        return {k: v for k, v in _attend("", op, batch, frames, heads, groups, dk, dv, dtype, op == "run" and rng.random() < 0.4,
                                         rng.random() < 0.5).items() if k != "name"}
    rows, cols = _log_int(rng, 1, 8192), _log_int(rng, 32, 4096)
    if rng.random() < 0.5:
        cols = max(32, cols // 32 * 32)
    if op == "norm":
        return {k: v for k, v in _norm("", rows, cols, dtype, rng.random() < 0.7).items() if k != "name"}
    outs = _log_int(rng, 16, 8192)
    return {k: v for k, v in _product("", op, rows, cols, outs, rng.choice(["mx4", "mx4", "mx8"]), dtype, rng.random() < 0.5).items() if k != "name"}


# ------------------------------------------------------------------------------------------ what a program has in hand
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Lengths of packed sequences: from the sizes alone, so that every seed has the same work; `frames` is their mean."""
    B, T = case["batch"], case["frames"]
    r = random.Random(1000 * B + T)
    w = [r.random() ** 2 + 0.02 for _ in range(B)]
    if B >= 4:
        w[B // 2] = 0.0
    total = B * T
    n = [int(total * x / sum(w)) for x in w]
    if B >= 4:
        n[B // 3] = 1
    n[max(range(B), key=lambda i: w[i])] += total - sum(n)
    return n


def _layout(x, fmt):
    """A matrix in the microscaled format (see above)."""
    rows, cols = x.shape
    groups, top = -(-cols // 32), 6.0 if fmt == "mx4" else 448.0
    y = torch.zeros(rows, groups * 32, dtype=torch.float32, device=x.device)
    y[:, :cols] = x.float()
    y = y.view(rows, groups, 32)
    most = y.abs().amax(-1)
    half, e = torch.frexp(most)                                    # most = half * 2^e, half in [0.5, 1)
    edge = 0.75 if fmt == "mx4" else 0.875                         # M = edge * 2^(3 or 9)
    k = e - (3 if fmt == "mx4" else 9) + (half > edge).int()
    k = torch.where(most > 0, k, torch.full_like(k, -127)).clamp_min(-127)
    y = torch.ldexp(y, -k.unsqueeze(-1))
    if fmt == "mx4":
        a = y.abs()
        code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) + 8 * (y < 0).to(torch.uint8)
        code = code.view(rows, groups * 16, 2)
        data = code[..., 0] | (code[..., 1] << 4)
    else:
        data = y.to(torch.float8_e4m3fn).view(torch.uint8).view(rows, groups * 32)
    tiles_r, tiles_g = -(-rows // 128), -(-groups // 4)
    s = torch.zeros(tiles_r * 128, tiles_g * 4, dtype=torch.uint8, device=x.device)
    s[:rows, :groups] = (k + 127).to(torch.uint8)
    s = s.view(tiles_r, 4, 32, tiles_g, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    return data.contiguous(), s


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    state = dict(case)
    if case["op"] in ("run", "step"):
        B, T, H, G, dk, dv = (case[k] for k in ("batch", "frames", "heads", "groups", "dk", "dv"))
        lead = (B,) if case["op"] == "step" else (B * T,) if case["packed"] else (T, B)
        state["q"] = torch.nn.functional.normalize(normal(*lead, H, dk), dim=-1).mul_(math.sqrt(dk)).to(dt)
        state["k"] = torch.nn.functional.normalize(normal(*lead, G, dk), dim=-1).to(dt)
        state["v"] = normal(*lead, G, dv).to(dt)
        if case["gated"]:                       # decays of a trained gate: mostly near 1, now and then a forgetful frame
            state["log_decay"] = torch.nn.functional.logsigmoid(3.0 + 1.5 * normal(*lead, G)) / 4
        else:                                   # time constants from 8 to 256 frames
            state["log_decay"] = -torch.exp2(-torch.linspace(3.0, 8.0, G, device=DEVICE))
        state["state"] = 0.5 * normal(B, G, dk, dv)
        state["scale"] = 1.0 / math.sqrt(dk)
        if case["packed"]:
            state["lengths"] = _lengths(case)
            state["offsets"] = torch.tensor([sum(state["lengths"][:i]) for i in range(B + 1)], dtype=torch.int64, device=DEVICE)
        return state
    if case["op"] in ("norm", "norm_product"):
        state["weight"] = 1.0 + 0.2 * normal(case["cols"])
        if case["op"] == "norm_product" or case["residual"]:
            state["added"] = normal(case["rows"], case["cols"]).to(dt)
    # features as a rectified layer's sums have them: a few channels much larger than the others
    state["x"] = (normal(case["rows"], case["cols"]) * torch.exp(0.7 * normal(case["cols"]))).to(dt)
    if case["op"] in ("product", "norm_product"):
        w = normal(case["outs"], case["cols"]) / math.sqrt(case["cols"])
        state["w_data"], state["w_scales"] = _layout(w, case["format"])
        state["bias"] = 0.1 * normal(case["outs"])
    return state


# ------------------------------------------------------------------------------------------ plain forms
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _values(data, scales, rows, cols, fmt):
    """The values that a microscaled matrix stands for, in 32 bits."""
    groups = -(-cols // 32)
    tiles_r, tiles_g = -(-rows // 128), -(-groups // 4)
    if fmt == "mx4":
        table = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), device=data.device)
        code = torch.stack((data & 15, data >> 4), dim=-1).view(rows, groups * 32)
        y = table[code.int()]
    else:
        y = data.view(torch.float8_e4m3fn).float().view(rows, groups * 32)
    s = scales.view(tiles_r, tiles_g, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(tiles_r * 128, tiles_g * 4)[:rows, :groups]
    return torch.ldexp(y.view(rows, groups, 32), (s.int() - 127).unsqueeze(-1)).view(rows, groups * 32)[:, :cols]


def _plain_norm(x, residual, weight):
    s = x.float() if residual is None else x.float() + residual.float()
    return s * torch.rsqrt(s.square().mean(-1, keepdim=True) + EPS) * weight, s


def _plain_product(x, s):
    a = _values(*_layout(x, s["format"]), s["rows"], s["cols"], s["format"])
    w = _values(s["w_data"], s["w_scales"], s["outs"], s["cols"], s["format"])
    y = torch.matmul(a, w.t()) + s["bias"]
    return (torch.relu(y) if s["relu"] else y).to(_dtype(s))


def _plain_run(s):
    """Chunks of 64 frames: products inside a chunk, sums of whole chunks, and those sums decayed to every later chunk."""
    B, T, H, G, dk, dv = (s[k] for k in ("batch", "frames", "heads", "groups", "dk", "dv"))
    C = 64
    q, k, v, g = s["q"], s["k"], s["v"], s["log_decay"]
    g = g if s["gated"] else g.expand(q.shape[:-2] + (G,))
    if s["packed"]:
        n = torch.tensor(s["lengths"], device=q.device)
        T = max(s["lengths"])
        at = torch.arange(T, device=q.device)[:, None]
        there = at < n                                             # [T][B]
        at = torch.where(there, at + s["offsets"][:-1], torch.zeros_like(at))
        q, k, v, g = (torch.where(there.view(T, B, *[1] * (x.dim() - 1)), x[at], torch.zeros_like(x[:1])) for x in (q, k, v, g))
    n_c = -(-T // C)

    def chunks(x):                                                 # [T][B][h][...] -> [B][h][n_c][C][...]
        x = x.movedim(0, 2)
        x = torch.cat((x, x.new_zeros(x.shape[:2] + (n_c * C - T,) + x.shape[3:])), dim=2)
        return x.reshape(x.shape[:2] + (n_c, C) + x.shape[3:])

    q, k, v = (chunks(x.float()) for x in (q, k, v))
    g = chunks(g.double()).cumsum(-1)                              # [B][G][n_c][C]: decay since the chunk's start
    whole = g[..., -1].cumsum(-1)                                  # decay up to each chunk's end
    local = torch.matmul((k * torch.exp(g[..., -1:] - g).float().unsqueeze(-1)).transpose(-1, -2), v)
    ends = torch.cat((torch.zeros_like(whole[..., :1]), whole), dim=-1)                          # [B][G][n_c + 1]
    far = torch.exp(torch.where(torch.ones(n_c + 1, n_c + 1, dtype=torch.bool, device=q.device).tril(), ends.unsqueeze(-1) - ends.unsqueeze(-2),
                                float("-inf"))).float()
    sums = torch.cat((s["state"].unsqueeze(2), local), dim=2)      # what enters at each chunk's end
    states = torch.matmul(far, sums.flatten(3)).view(B, G, n_c + 1, dk, dv)
    last = states[:, :, -1].contiguous()
    q = q.view(B, G, H // G, n_c, C, dk)
    mask = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    near = torch.exp(torch.where(mask, g.unsqueeze(-1) - g.unsqueeze(-2), float("-inf"))).float()
    p = torch.matmul(q, k.unsqueeze(2).transpose(-1, -2)) * near.unsqueeze(2)
    o = torch.matmul(p, v.unsqueeze(2)) + torch.exp(g).float()[:, :, None, :, :, None] * torch.matmul(q, states[:, :, None, :-1])
    o = (s["scale"] * o).to(_dtype(s)).view(B, H, n_c * C, dv)[:, :, :T].movedim(2, 0)           # [T][B][H][dv]
    if s["packed"]:
        out = torch.zeros_like(s["q"][..., :1]).repeat(1, 1, dv)
        out[at[there]] = o[there]
        return out, last
    return o.contiguous(), last


def _plain_step(s):
    B, H, G, dk, dv = (s[k] for k in ("batch", "heads", "groups", "dk", "dv"))
    g = s["log_decay"].expand(B, G)
    new = torch.exp(g)[..., None, None] * s["state"] + s["k"].float().unsqueeze(-1) * s["v"].float().unsqueeze(-2)
    o = s["scale"] * torch.matmul(s["q"].float().view(B, G, H // G, dk), new)
    s["state"].copy_(new)
    return o.to(_dtype(s)).view(B, H, dv), s["state"]


def run(state):
    s = state
    if own:
        from paper_1806_04965_b200 import Microscaled, linear_attention_run, linear_attention_step, product, quantize, rms_norm
        if s["op"] == "run":
            return linear_attention_run(s["q"], s["k"], s["v"], s["log_decay"], state=s["state"], offsets=s.get("offsets"), scale=s["scale"])
        if s["op"] == "step":
            return linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], scale=s["scale"]), s["state"]
        if s["op"] == "norm":
            return rms_norm(s["x"], s["weight"], residual=s.get("added"), eps=EPS)
        w = Microscaled(s["w_data"], s["w_scales"], s["outs"], s["cols"], s["format"])
        if s["op"] == "product":
            return product(quantize(s["x"], s["format"]), w, bias=s["bias"], relu=s["relu"], dtype=s["x"].dtype)
        a, total = rms_norm(s["x"], s["weight"], residual=s["added"], eps=EPS, format=s["format"])
        return product(a, w, bias=s["bias"], relu=s["relu"], dtype=s["x"].dtype), total
    if s["op"] == "run":
        return _plain_run(s)
    if s["op"] == "step":
        return _plain_step(s)
    if s["op"] == "norm":
        y, total = _plain_norm(s["x"], s.get("added"), s["weight"])
        y = y.to(_dtype(s))
        return y if s.get("added") is None else (y, total.to(_dtype(s)))
    if s["op"] == "product":
        return _plain_product(s["x"], s)
    y, total = _plain_norm(s["x"], s["added"], s["weight"])
    return _plain_product(y, s), total.to(_dtype(s))


# ------------------------------------------------------------------------------------------ work, and the definitions in 64 bits
def work(case):
    el = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("run", "step"):
        B, T, H, G, dk, dv = (case[k] for k in ("batch", "frames", "heads", "groups", "dk", "dv"))
        n = B * T
        n_bytes = n * el * (H * dk + G * dk + G * dv + H * dv) + 2 * 4 * B * G * dk * dv + 4 * (n * G if case["gated"] else G)
        return {"bytes": n_bytes, "flops": n * 2 * dk * dv * (G + H)}
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "norm":
        return {"bytes": rows * cols * el * (4 if case["residual"] else 2) + 4 * cols, "flops": 5 * rows * cols}
    held = (0.5 if case["format"] == "mx4" else 1.0) + 1 / 32
    n_bytes = rows * cols * el * (3 if case["op"] == "norm_product" else 1) + case["outs"] * cols * held + rows * case["outs"] * el + 4 * case["outs"]
    return {"bytes": n_bytes, "flops": 2 * rows * cols * case["outs"]}


def _exact_round(x, fmt):
    """x rounded to the microscaled format, as values in 64 bits."""
    rows, cols = x.shape
    pad = -cols % 32
    y = torch.nn.functional.pad(x, (0, pad)).reshape(rows, -1, 32)
    most = y.abs().max(dim=-1, keepdim=True).values / (6.0 if fmt == "mx4" else 448.0)
    m, e = torch.frexp(most)
    unit = torch.ldexp(torch.ones_like(m), torch.where(m > 0.5, e, e - 1))
    unit = torch.where(most > 0, unit, torch.ones_like(unit)).clamp_min(2.0 ** -127)
    y = y / unit
    bits, low = (1, 0) if fmt == "mx4" else (3, -6)                # digits behind the point, smallest exponent of the elements
    _, e = torch.frexp(y)
    grid = torch.ldexp(torch.ones_like(y), (e - 1).clamp_min(low) - bits)
    return (torch.round(y / grid) * grid * unit).reshape(rows, -1)[:, :cols]


def _exact_weights(s):
    rows, cols, fmt = s["outs"], s["cols"], s["format"]
    r = torch.arange(rows, device=s["w_data"].device)[:, None]
    c = torch.arange(cols, device=s["w_data"].device)[None, :]
    g = c // 32
    k = s["w_scales"][(r // 128 * (-(-cols // 128)) + g // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + g % 4].double() - 127
    if fmt == "mx4":
        code = (s["w_data"].long()[r, c // 2] >> (4 * (c % 2))) & 15
        e, m = (code >> 1) & 3, code & 1
        y = torch.where(e == 0, m * 0.5, (1 + 0.5 * m) * torch.exp2(e.double() - 1))
        y = torch.where(code >= 8, -y, y)
    else:
        code = s["w_data"].long()[r, c]
        e, m = (code >> 3) & 15, code & 7
        y = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2(e.double() - 7))
        y = torch.where(code >= 128, -y, y)
    return y * torch.exp2(k)


def _exact_attention(s):
    """Frame by frame, as the recurrence is written."""
    G, H = s["groups"], s["heads"]
    packed = s["op"] == "run" and s["packed"]
    lead = s["q"].shape[:-2]
    d = torch.exp(s["log_decay"].double()).expand(lead + (G,))
    q, k, v = (s[x].double() for x in ("q", "k", "v"))
    S = s["state"].double().clone()
    out = torch.zeros(lead + (H, s["dv"]), dtype=torch.float64, device=q.device)

    def frame(S, q, k, v, d):
        S = S * d[..., None, None] + torch.einsum("bgi,bgj->bgij", k, v)
        return S, s["scale"] * torch.einsum("bghi,bgij->bghj", q.unflatten(1, (G, H // G)), S).flatten(1, 2)

    if s["op"] == "step":
        S, o = frame(S, q, k, v, d)
        return o, S
    if not packed:
        for t in range(s["frames"]):
            S, out[t] = frame(S, q[t], k[t], v[t], d[t])
        return out, S
    first = [sum(s["lengths"][:i]) for i in range(s["batch"])]
    order = sorted(range(s["batch"]), key=lambda b: -s["lengths"][b])
    index = torch.tensor(order, device=q.device)
    at = torch.tensor([first[b] for b in order], device=q.device)
    S = S[index]
    n = len(order)
    for t in range(max(s["lengths"])):
        while n and s["lengths"][order[n - 1]] <= t:
            n -= 1
        i = at[:n] + t
        S[:n], out[i] = frame(S[:n], q[i], k[i], v[i], d[i])
    back = torch.empty_like(S)
    back[index] = S
    return out, back


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] in ("run", "step"):
        return _exact_attention(s)
    x = s["x"].double()
    if s["op"] != "product":
        total = x + s["added"].double() if "added" in s else x
        x = total / torch.sqrt((total * total).sum(-1, keepdim=True) / s["cols"] + EPS) * s["weight"].double()
        if s["op"] == "norm":
            return (x, total) if "added" in s else x
    y = torch.matmul(_exact_round(x, s["format"]), _exact_weights(s).t()) + s["bias"].double()
    y = y.clamp_min(0) if s["relu"] else y
    return y if s["op"] == "product" else (y, total)
