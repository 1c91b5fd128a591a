"""Block norm where a CTA or a cluster takes many rows one after the other: the exchange areas of its sums alternate over
turns, and the column sums add up over them.  Tolerances as in test_gpu_training.py.
"""
import pytest
import torch

import paper_1801_00829_b200 as fo
from test_gpu_training import BF16, F16, F32, F64, Case

pytestmark = pytest.mark.gpu


def both_ways(c):
    h, y, stats = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    return [h, y, stats] + list(fo.fused_block_norm_grad(c.dh, c.dy, h, c.f, stats, **c.how()).values())


@pytest.mark.parametrize("cols", [8192, 16384, 20000, 32768, 9001])
@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, BF16), (F32, F32)])
def test_rows_over_clusters(stream, block, cols):
    """Rows of 8193 columns and more are spread over 2 or 4 CTAs, the gradient's of 4097 and more over 2, 4 or 8."""
    c = Case(333, cols, stream, block, "layer", "col", "sigmoid", "layer", bias=True)
    c.check_backward(*c.check_forward())


@pytest.mark.parametrize("cols", [8192, 16384, 32768])
def test_rows_over_clusters_in_the_short_form(cols):
    c = Case(333, cols, BF16, BF16, "rms", "cell", "sigmoid", "rms")
    c.check_backward(*c.check_forward())


def test_rows_over_clusters_in_64_bits():
    c = Case(301, 8194, F64, F64, "layer", "row", "tanh", "rms", bias=True)
    c.check_backward(*c.check_forward())


def test_rows_over_clusters_one_call_behind_the_other():
    """Every call starts while the one before it ends."""
    c = Case(40, 16384, F16, F16, "layer", None, "linear", "layer")
    first = both_ways(c)
    for _ in range(20):
        again = both_ways(c)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("cols", [96, 1000, 1001, 4096, 9000])
def test_the_result_of_one_call_as_a_vector_of_the_next(cols):
    """Each call starts while the one before it ends, and takes its result as a gate, a scale and a weight."""
    torch.manual_seed(3)
    x, f = torch.randn(64, cols, device="cuda"), torch.randn(64, cols, device="cuda")
    seeds = torch.rand(12, cols, device="cuda") + 0.5
    v, w = torch.empty(1, cols, device="cuda"), torch.empty(1, cols, device="cuda")

    def chain(between):
        out = []
        for k in range(12):
            fo.fused_block_norm(seeds[k:k + 1], pre=("rms", None, None, 1e-6), out_y=v)
            between()
            fo.fused_block_norm(seeds[k:k + 1], pre=("layer", v[0], None, 1e-6), out_y=w)
            between()
            h, y, stats = fo.fused_block_norm(x, f, post=("rms", v[0], None, 1e-6), gate=("col", w[0], "sigmoid"), col_scale=v[0],
                                              pre=("rms", w[0], None, 1e-6), stats=True)
            between()
            got = fo.fused_block_norm_grad(h, y, h, f, stats, post=("rms", v[0], None, 1e-6), gate=("col", w[0], "sigmoid"),
                                           col_scale=v[0], pre=("rms", w[0], None, 1e-6))
            between()
            out += [h, y] + list(got.values())
        return out

    want = chain(torch.cuda.synchronize)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(want, chain(lambda: None)))
