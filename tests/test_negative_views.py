"""Tensors that are views with the negative bit set, as the imaginary part of a conjugate is: what lies in memory has the other sign, and
the operators, which read memory, refuse them (no GPU needed)."""
import pytest
import torch

import paper_1801_00829_b200 as fo

X = torch.complex(torch.zeros(6, 8), torch.ones(6, 8)).conj().imag


def test_it_is_such_a_view():
    assert X.is_neg() and (X == -1.0).all()


@pytest.mark.parametrize("call", [
    lambda x, y: fo.fused_head_norm(x.view(1, 6, 8)), lambda x, y: fo.fused_head_norm(y.view(1, 6, 8), x.view(1, 6, 8)),
    lambda x, y: fo.fused_head_norm_grad(x.view(1, 6, 8)),
    lambda x, y: fo.fused_scan(x, y), lambda x, y: fo.fused_scan_grad(y, y, x, y), lambda x, y: fo.fused_distill(x, y.long(), y),
    lambda x, y: fo.fused_distill_grad(None, x, y.long(), y, y), lambda x, y: fo.fused_distill_step(None, x, y.long(), y),
    lambda x, y: fo.fused_block_norm(x, None, pre=("rms", None, None, 1e-6)),
], ids=range(9))
def test_refused(call):
    with pytest.raises(ValueError, match="negative view"):
        call(X, torch.zeros(6, 8))
