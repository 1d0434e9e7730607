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
