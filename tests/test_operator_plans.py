"""How products and runs are cut on a device of 148 SMs, and that the GPU tests of test_gpu_operator_borders.py take every path there is."""
import math
import random

import pytest
import torch

from paper_1806_04965_b200 import SrError, operators as ops

SMS = 148
# rows, cols, outs, format, (rows of a tile, CTAs that share a reduction, pairs): one for each path, found by a search for small ones
PRODUCTS = [
    (2, 33, 131, "mx4", (16, 1, 0)), (2, 35, 130, "mx8", (16, 1, 0)), (2, 260, 131, "mx4", (16, 2, 0)), (2, 130, 133, "mx8", (16, 2, 0)),
    (5, 769, 132, "mx4", (16, 4, 0)), (1, 386, 133, "mx8", (16, 4, 0)), (2, 1804, 138, "mx4", (16, 8, 0)), (3, 897, 130, "mx8", (16, 8, 0)),
    (17, 35, 130, "mx4", (32, 1, 0)), (18, 34, 132, "mx8", (32, 1, 0)), (17, 807, 4840, "mx4", (32, 2, 0)), (27, 392, 4781, "mx8", (32, 2, 0)),
    (32, 784, 136, "mx4", (32, 4, 0)), (30, 388, 130, "mx8", (32, 4, 0)), (32, 1793, 150, "mx4", (32, 8, 0)), (17, 901, 145, "mx8", (32, 8, 0)),
    (36, 33, 136, "mx4", (64, 1, 0)), (37, 38, 131, "mx8", (64, 1, 0)), (1189, 1802, 131, "mx4", (64, 2, 0)), (785, 944, 276, "mx8", (64, 2, 0)),
    (36, 1315, 133, "mx4", (64, 4, 0)), (39, 646, 136, "mx8", (64, 4, 0)), (47, 1799, 151, "mx4", (64, 8, 0)), (40, 904, 135, "mx8", (64, 8, 0)),
    (1160, 33, 900, "mx4", (128, 1, 0)), (918, 33, 1158, "mx8", (128, 1, 0)), (199, 7950, 2393, "mx4", (128, 2, 0)), (74, 4010, 4870, "mx8", (128, 2, 0)),
    (811, 8811, 265, "mx4", (128, 4, 0)), (1229, 4631, 138, "mx8", (128, 4, 0)), (66, 17540, 1293, "mx4", (128, 8, 0)), (66, 8782, 1154, "mx8", (128, 8, 0)),
    (1548, 36, 1416, "mx4", (192, 1, 0)), (1559, 34, 1451, "mx8", (192, 1, 0)), (4768, 1867, 387, "mx4", (192, 1, 1)), (2689, 916, 778, "mx8", (192, 1, 1)),
    (4807, 8808, 136, "mx4", (192, 2, 0)), (5120, 3793, 149, "mx8", (192, 2, 0)), (2610, 6993, 148, "mx4", (192, 4, 0)), (2781, 3476, 134, "mx8", (192, 4, 0)),
    (1274, 11615, 148, "mx4", (192, 8, 0)), (1368, 5837, 136, "mx8", (192, 8, 0)),
]
# lengths, heads, groups, dk, dv, frames of a segment: packed bf16 sequences that are cut into segments, with sequences of none, one, exactly a segment's and one more frames, more than 32 sequences
S = 512
RUNS = [
    ([5000, 0, 1, S, S + 1, 2986], 2, 1, 64, 64, S),
    ([0, 3000, S, 2 * S + 1, 1464], 4, 2, 128, 72, S),
    ([8000, 0, 700] + [1, 0, 5, 128, 129] * 7 + [S, S + 1, 2 * S, 3000], 4, 2, 40, 64, S),
    ([1280, 641, 4255], 3, 3, 96, 200, 640),
]


def plan(rows, cols, outs, fmt, sms=SMS):
    p = ops.product_plan(rows, cols, outs, fmt, sms)
    return p["rows"], p["parts"], p["pair"]


def test_every_way_to_cut_a_product_is_in_the_list():
    for rows, cols, outs, fmt, want in PRODUCTS:
        assert plan(rows, cols, outs, fmt) == want, (rows, cols, outs, fmt)
    rng, seen = random.Random(7), set()

    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    for _ in range(30000):
        fmt = rng.choice(["mx4", "mx8"])
        seen.add((fmt, plan(size(1, 16384), size(1, 32768), size(1, 32768), fmt)))
    assert seen <= {(fmt, want) for _, _, _, fmt, want in PRODUCTS}


def test_packed_runs_in_the_list_are_cut():
    for lengths, heads, groups, dk, dv, segment in RUNS:
        p = ops.attention_plan(torch.bfloat16, len(lengths), sum(lengths), heads, groups, dk, dv, packed=True, sms=SMS)
        assert p["chunk"] == 128 and p["segment"] == segment, (p, len(lengths))
        assert p["segments"] >= sum(max(1, -(-n // segment)) for n in lengths)
    assert max(len(r[0]) for r in RUNS) > 32
    whole = ops.attention_plan(torch.bfloat16, 37, 4096, 2, 2, 128, 128, sms=SMS)
    assert whole == {"chunk": 128, "segment": 0, "segments": 0}
    assert ops.attention_plan(torch.float32, 1, 5000, 1, 1, 64, 64, sms=SMS)["chunk"] == 16


def test_plans_refuse():
    for bad in ((0, 32, 32, "mx4"), (4, 0, 32, "mx4"), (4, 32, 0, "mx4"), (4, 32, 32, "mx6"), (1 << 31, 32, 32, "mx4")):
        with pytest.raises(SrError):
            ops.product_plan(*bad, SMS)
    with pytest.raises(SrError):
        ops.product_plan(4, 32, 32, "mx4", -1)
    with pytest.raises(SrError):
        ops.attention_plan(torch.bfloat16, 1, 100, 1, 1, 300, 64, sms=SMS)
