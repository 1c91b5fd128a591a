"""Calls of the head norms, the recurrence and the distillation loss at the edges of what they allow.  Tolerances as in test_gpu_lm.py
where nothing else is said."""
import numpy as np
import pytest
import torch

import paper_1801_00829_b200 as fo
from test_gpu_lm import BF16, F16, F32, F64, PAIRS, TYPES, Distill, Heads, close, host, ref, unit, wide

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------ head norms
def many_tokens(dtype, pairing):
    """A warp's groups take a token each, and the last warp has fewer tokens than groups."""
    return Heads(1, 4003, 7, 3, 64, 48, dtype, pairing, "rms", bias=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", ["halves", "pairs"])
def test_heads_of_tables_without_rows(dtype, pairing):
    """Every position is outside: what is turned is NaN, the rest as without a rotation."""
    c = many_tokens(dtype, pairing)
    cos, sin = c.rotate[:2]
    c.rotate = (cos[:0], sin[:0]) + c.rotate[2:]
    c.check()
    assert torch.isnan(fo.fused_head_norm(c.q, c.k, **c.how())[0][..., :48]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", ["halves", "pairs"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_heads_beside_a_table_row_that_no_token_uses(dtype, pairing, bad):
    c = many_tokens(dtype, pairing)
    c.positions.clamp_(min=1)
    want = list(fo.fused_head_norm(c.q, c.k, **c.how()))
    grads = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how())
    for t in c.rotate[:2]:
        t[0] = bad
    got = fo.fused_head_norm(c.q, c.k, **c.how())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how())
    assert all(torch.equal(got[k], grads[k]) for k in grads)
