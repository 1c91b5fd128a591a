"""Block norm where a CTA or a cluster takes many rows one after the other: the exchange areas of its sums alternate over
turns, and the column sums add up over them.  Tolerances as in test_gpu_training.py.
"""
import threading

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


@pytest.mark.parametrize("rows,cols", [(700, 4096), (1300, 2048), (5000, 128), (9001, 64)])
@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, F16)])
@pytest.mark.parametrize("gate", ["cell", None])
def test_the_short_form_over_many_rows(rows, cols, stream, block, gate):
    """Root-mean-square norms with weights and without biases, a gate per element: several rows for every CTA."""
    c = Case(rows, cols, stream, block, "rms", gate, "sigmoid" if gate else "linear", "rms", wide=stream == F32)
    c.check_backward(*c.check_forward())


def test_two_threads():
    """Calls from two threads, on streams of their own and on one they share."""
    cases = [Case(400, 1000, BF16, BF16, "layer", "cell", "silu", "layer", seed=s) for s in (1, 2)]
    grads = [[torch.full((n,), float(s), device="cuda") for n in (4000, 77)] for s in (1, 2)]
    want = [both_ways(c) + [fo.fused_grad_norm(g, 1.0)] for c, g in zip(cases, grads)]
    torch.cuda.synchronize()
    shared = torch.cuda.Stream()
    for streams in ((torch.cuda.Stream(), torch.cuda.Stream()), (shared, shared)):
        wrong, errors = [], []

        def work(k):
            try:
                with torch.cuda.stream(streams[k]):
                    for _ in range(30):
                        got = both_ways(cases[k]) + [fo.fused_grad_norm(grads[k], 1.0)]
                        streams[k].synchronize()
                        wrong.extend(1 for a, b in zip(got, want[k]) if not torch.equal(a, b))
            except Exception as e:  # noqa: BLE001
                errors.append(e)

        threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors and not wrong


def test_nothing_is_allocated_by_the_library():
    """Device memory after calls with results and scratch in place is what it was: only kernels are launched."""
    c = Case(300, 1000, BF16, BF16, "rms", "cell", "sigmoid", "rms")
    out_h, out_y = torch.empty_like(c.x), torch.empty(300, 1000, dtype=BF16, device="cuda")
    grads = [torch.rand(n, device="cuda") for n in (100000, 77)]
    p, m, v = ([torch.rand(n, device="cuda") for n in (100000, 77)] for _ in range(3))
    kept, adam = fo.tensor_list(grads), fo.adam_list(p, grads, m, v)

    def calls():
        _, _, stats = fo.fused_block_norm(c.x, c.f, out_h=out_h, out_y=out_y, stats=True, **c.how())
        fo.fused_block_norm_grad(c.dh, c.dy, out_h, c.f, stats, **c.how())
        fo.fused_adamw(adam, lr=0.1, factor=fo.fused_grad_clip(kept, 1.0)[1:])

    for _ in range(3):                                       # kernels are loaded, torch's own cache is filled
        calls()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(50):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
