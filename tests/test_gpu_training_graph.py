"""The training-step operators captured into a CUDA graph: the graph's scratch is its own, so that calls outside it, on the
same stream too, and the graph do not touch each other's."""
import pytest
import torch

import paper_1801_00829_b200 as fo
from test_gpu_training import BF16, Case

pytestmark = pytest.mark.gpu


def step(c, grads, clipped, adam):
    """Everything once: block norm, its gradient, clipping into other tensors, an update in place."""
    h, y, stats = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    got = fo.fused_block_norm_grad(c.dh, c.dy, h, c.f, stats, **c.how())
    result = fo.fused_grad_clip(fo.tensor_list(grads, clipped), 0.5)
    fo.fused_adamw(adam, lr=0.01, step=3, factor=result[1:])
    return [h, y, stats, result] + [got[k] for k in sorted(got)]


def state(seed):
    torch.manual_seed(seed)
    sizes = (4099, 64, 30000)
    grads = [torch.randn(n, device="cuda") for n in sizes]
    p, m, v = ([torch.rand(n, device="cuda") for n in sizes] for _ in range(3))
    return grads, [torch.zeros(n, device="cuda") for n in sizes], p, m, v


def test_captured_and_replayed():
    c = Case(67, 1000, BF16, BF16, "layer", "col", "sigmoid", "rms", bias=True)
    grads, clipped, p, m, v = state(5)
    adam = fo.adam_list(p, grads, m, v)
    start = [t.clone() for t in (*p, *m, *v)]

    def rewind():
        for t, s in zip((*p, *m, *v), start):
            t.copy_(s)

    want = [t.clone() for t in step(c, grads, clipped, adam)]
    after = [t.clone() for t in (*clipped, *p, *m, *v)]
    rewind()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(c, grads, clipped, adam)
    # calls outside the graph on the captured stream, before it has ever run, and larger ones, which take more scratch
    big = Case(700, 4096, BF16, BF16, "rms", "cell", "sigmoid", "rms")
    other = [torch.full((50000,), 2.0, device="cuda")]
    here = [t.clone() for t in both(big)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm = fo.fused_grad_norm(other, 1.0, result_type=torch.float64)
        there = both(big)
    torch.cuda.synchronize()
    assert norm[0].item() == pytest.approx(2.0 * 50000 ** 0.5, rel=1e-6)
    assert all(torch.equal(a, b) for a, b in zip(here, there))
    for _ in range(3):
        for t in (*got, *clipped):
            t.zero_()
        rewind()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert all(torch.equal(a, b) for a, b in zip(after, (*clipped, *p, *m, *v)))


def both(c):
    h, y, stats = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    return [h, y, stats] + list(fo.fused_block_norm_grad(c.dh, c.dy, h, c.f, stats, **c.how()).values())


def test_a_captured_template_operator():
    """The same for an operator of the templates (its scratch comes from the same place)."""
    x = torch.rand(300, 70, dtype=torch.float64, device="cuda")
    want = fo.fused_cell([("sq", "t0", "a")], "t0", x, agg="full").clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = fo.fused_cell([("sq", "t0", "a")], "t0", x, agg="full")
    with torch.cuda.stream(side):
        first = fo.fused_cell([("sq", "t0", "a")], "t0", x, agg="full")
    torch.cuda.synchronize()
    assert torch.equal(first, want)
    for _ in range(2):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
