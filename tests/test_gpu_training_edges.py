"""Results of the training-step operators that are easily left out: sums over nothing, gradients of arguments that were not
given, values at the ends of the range.  Tolerances as in test_gpu_training.py."""
import numpy as np
import pytest
import torch

import paper_1801_00829_b200 as fo
from oracle import training as ref
from paper_1801_00829_b200.binding import workspace
from test_gpu_training import BF16, F16, F32, F64, Case, close, host, unit
from test_training_abi import BLOCK_NORM_GRAD, NONE

pytestmark = pytest.mark.gpu

CODE = {F64: 0, F32: 1, BF16: 2, F16: 3}


@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, F16), (F64, F64)])
@pytest.mark.parametrize("gate", [None, "cell", "row", "col"])
@pytest.mark.parametrize("rows,cols", [(19, 130), (7, 1001)])
def test_gradient_of_a_column_scale_that_is_not_there(stream, block, gate, rows, cols):
    """The C call: dcol_scale with col_scale NULL is the gradient at a scale of ones."""
    c = Case(rows, cols, stream, block, "rms", gate, "silu" if gate else "linear", None, col_scale=False)
    _, _, stats = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    wide = F64 if block == F64 else F32
    got = torch.full((cols,), float("nan"), dtype=wide, device="cuda")
    lib = fo.load_library()
    need = lib.fused_block_norm_grad_workspace_bytes(rows, cols, CODE[block])
    ws = workspace(c.f.device, need)
    access = {None: 0, "cell": 0, "row": 1, "col": 2}[gate]
    g = c.gate[1] if gate else None
    post = (1, 0, c.post[3], c.post[1].data_ptr(), 0)
    types = CODE[stream], CODE[block], CODE[block]
    packed = BLOCK_NORM_GRAD.pack(rows, cols, *types, access, 2 if gate else 0, 0, c.dh.data_ptr(), 0, 0,
                                  c.f.data_ptr(), g.data_ptr() if gate else 0, 0, stats.data_ptr(), c.dh.stride(0), 0, 0,
                                  c.f.stride(0), g.stride(0) if gate else 0, c.scale, *post, *NONE, 0, 0, 0, 0, 0, 0,
                                  got.data_ptr(), 0, 0, 0, 0)
    st = torch.cuda.current_stream().cuda_stream
    assert lib.fused_block_norm_grad(packed, ws.data_ptr(), ws.numel(), st) == 0
    want = ref.block_norm_grad(host(c.dh), None, None, host(c.f), host(stats), **c.host_how())["col_scale"]
    close(got, *want, unit(block), "dcol_scale", rows=max(rows, cols))


def leave_garbage(*shapes):
    """Memory that the next tensors of these sizes are likely to get, full of NaN."""
    for s in shapes:
        torch.full(s, float("nan"), device="cuda")


@pytest.mark.parametrize("block", [F32, BF16])
def test_rows_without_columns(block):
    """Sums over no columns are zero: the gradient of a gate per row, and the statistics."""
    x = torch.zeros(300, 0, dtype=block, device="cuda")
    g = torch.ones(300, dtype=block, device="cuda")
    for _ in range(3):
        leave_garbage((300,), (4, 300))
        h, _, stats = fo.fused_block_norm(x, x, post=("rms", None, None, 1e-6), gate=("row", g, "silu"), stats=True)
        assert bool((stats == 0).all())
        leave_garbage((300,), (4, 300))
        got = fo.fused_block_norm_grad(h, None, None, x, stats, post=("rms", None, None, 1e-6), gate=("row", g, "silu"))
        assert got["gate"].shape == (300,) and bool((got["gate"] == 0).all())


@pytest.mark.parametrize("stream,block", [(F32, F32), (BF16, BF16), (F32, F16), (F64, F64)])
@pytest.mark.parametrize("where", ["post", "col_scale", "gate"])
@pytest.mark.parametrize("cols", [5, 100, 1000, 1001, 4104, 9000])
def test_an_infinite_factor_stays_in_its_column(stream, block, where, cols):
    """An infinite weight, column scale or gate in the last piece of rows that leave threads without elements: h is
    infinite in that column, r is 0 and y is 0 in all others."""
    c = Case(3, cols, stream, block, "rms", "col", "linear", "rms")
    factor = {"post": c.post[1], "col_scale": c.col_scale, "gate": c.gate[1]}[where]
    factor[cols - 1] = float("inf")
    h, y, stats = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    assert bool(torch.isinf(h[:, -1]).all()) and bool(torch.isfinite(h[:, :-1]).all())
    assert bool((y[:, :-1] == 0).all()) and bool(torch.isnan(y[:, -1]).all())
    assert bool((stats[3] == 0).all()) and bool(torch.isfinite(stats).all())


def gate_parts(act, g):
    """act(g), act'(g) and the magnitude act' is added up from, in float64 and without a difference that cancels."""
    if act == "tanh":
        q = np.exp(-2.0 * np.abs(g))
        return np.tanh(g), 4.0 * q / (1.0 + q) ** 2, 4.0 * q / (1.0 + q) ** 2
    e = np.exp(-np.abs(g))
    small, large = e / (1.0 + e), 1.0 / (1.0 + e)
    s, rest = np.where(g < 0, small, large), np.where(g < 0, large, small)
    if act == "sigmoid":
        return s, s * rest, s * rest
    return g * s, s * (1.0 + g * rest), s * (1.0 + np.abs(g) * rest)


PAIRS = [(F64, F64), (F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)]


def gates(n, block, least=-40.0, most=40.0):
    return torch.linspace(least, most, n, dtype=torch.float64).to(block).cuda()


@pytest.mark.parametrize("stream,block", PAIRS)
@pytest.mark.parametrize("act", ["sigmoid", "silu", "tanh"])
@pytest.mark.parametrize("cols", [256, 1001])
def test_slopes_of_open_and_closed_gates(stream, block, act, cols):
    """The gate's gradient relative to act'(g) itself: the slope of an open gate is a small number, not the difference of
    two that are near 1.  Its factors: an exponential, a sum, a reciprocal and at most six products, within 64 rounding
    units together."""
    c = Case(5, cols, stream, block, None, None, "linear", None, col_scale=False)
    g = gates(5 * cols, block).reshape(5, cols)
    got = fo.fused_block_norm_grad(c.dh, None, None, c.f, None, gate=("cell", g, act), scale=c.scale)
    qz = host(c.dh) * c.scale * host(c.f)
    _, slope, size = gate_parts(act, host(g))
    close(got["gate"], qz * slope, np.abs(qz) * size, unit(block), "gate")


@pytest.mark.parametrize("stream,block", PAIRS)
@pytest.mark.parametrize("act", ["sigmoid", "silu", "tanh"])
@pytest.mark.parametrize("access", ["row", "col"])
def test_slopes_of_shared_gates(stream, block, act, access):
    """A gate per row or column has its gradient in 32 bits (64): as many more units as terms are added."""
    rows, cols = (300, 65) if access == "row" else (9, 300)
    c = Case(rows, cols, stream, block, None, None, "linear", None, col_scale=False)
    g = gates(300, block)
    got = fo.fused_block_norm_grad(c.dh, None, None, c.f, None, gate=(access, g, act), scale=c.scale)
    qz = host(c.dh) * c.scale * host(c.f)
    _, slope, size = gate_parts(act, host(g)[:, None] if access == "row" else host(g))
    axis = 1 if access == "row" else 0
    close(got["gate"], (qz * slope).sum(axis=axis), (np.abs(qz) * size).sum(axis=axis), unit(block), "gate",
          rows=qz.shape[axis])


@pytest.mark.parametrize("stream,block", [(F32, F32), (F32, BF16), (F32, F16)])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("access", ["cell", "row", "col"])
def test_a_32_bit_stream_gets_32_bit_gates(stream, block, act, access):
    """h in 32 bits, gate values of 4 to 60 in magnitude: the activation is an exponential within 2^-22 (four rounding
    units), a sum and a reciprocal (three units), and h takes four more products: 16 units hold all of it."""
    rows, cols = 40, 264
    c = Case(rows, cols, stream, block, None, None, "linear", None, col_scale=False)
    n = {"cell": rows * cols, "row": rows, "col": cols}[access]
    g = gates(n, block, -60.0, 60.0)
    g = g.reshape(rows, cols) if access == "cell" else g
    h, _, _ = fo.fused_block_norm(torch.zeros(rows, cols, device="cuda"), c.f, gate=(access, g, act), scale=c.scale)
    a, _, _ = gate_parts(act, host(g)[:, None] if access == "row" else host(g))
    want = host(c.f) * c.scale * a
    assert h.dtype == F32 and np.all(np.abs(host(h) - want) <= 16 * 2.0 ** -24 * np.abs(want))


@pytest.mark.parametrize("block", [BF16, F16])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("access", ["cell", "row", "col"])
def test_summed_gradients_get_32_bit_gates(block, act, access):
    """The gradient of a column scale is in 32 bits beside 16-bit blocks: one row, so that its only term is seen.  As
    above, two products more."""
    cols = 264
    c = Case(1, cols, block, block, None, None, "linear", None)
    for value in (-60.0, -25.5, -11.25, -4.5, 4.5, 30.0):
        g = torch.full((1, cols) if access == "cell" else (1,) if access == "row" else (cols,), value, dtype=block, device="cuda")
        got = fo.fused_block_norm_grad(c.dh, None, None, c.f, None, gate=(access, g, act), scale=c.scale, col_scale=c.col_scale)
        want = (host(c.dh) * c.scale * host(c.f) * gate_parts(act, np.full((1, cols), value))[0])[0]
        assert np.all(np.abs(host(got["col_scale"]) - want) <= 18 * 2.0 ** -24 * np.abs(want)), value


@pytest.mark.parametrize("stream,block", PAIRS)
@pytest.mark.parametrize("act", ["sigmoid", "silu", "tanh"])
def test_gates_at_the_ends_of_the_range(stream, block, act):
    """Gates of the type's largest values, infinities and NaN: a closed gate lets nothing through, and an open one's slope
    is nothing (SiLU's is one)."""
    top = torch.finfo(block).max
    values = torch.tensor([-top, -1e4, -200.0, 200.0, 1e4, top, float("inf"), float("-inf"), float("nan")], dtype=torch.float64)
    g = values.to(block).cuda()
    x = torch.zeros(4, 9, dtype=stream, device="cuda")
    f = torch.ones(4, 9, dtype=block, device="cuda")
    h, _, _ = fo.fused_block_norm(x, f, gate=("col", g, act))
    got = fo.fused_block_norm_grad(torch.ones_like(x), None, None, f, None, gate=("col", g, act))
    a, slope = host(h)[0], host(got["gate"])
    assert np.isnan(a[8]) and np.isnan(slope[8]) and np.array_equal(host(got["f"])[0], a, equal_nan=True)
    none = 1e4 * np.exp(-200.0)                             # what +-200 leave in float64; less than 32 bits hold
    closed = {"sigmoid": [0, 1, 2, 7], "silu": [0, 1, 2], "tanh": []}[act]
    assert (np.abs(a[closed]) <= none).all()
    if act == "tanh":
        assert a[:8].tolist() == [-1, -1, -1, 1, 1, 1, 1, -1]
    else:
        assert a[3:7].tolist() == ([1.0] * 4 if act == "sigmoid" else host(g)[3:7].tolist())
    flat = [0, 1, 2] if act == "silu" else list(range(8))
    assert (np.abs(slope[flat]) <= none).all() and (act != "silu" or (slope[3:6] == 4.0).all())


@pytest.mark.parametrize("block", [BF16, F16])
@pytest.mark.parametrize("mode", [("rms", "cell", "sigmoid", "rms"), (None, "row", "silu", "layer"), ("layer", None, "linear", None)])
@pytest.mark.parametrize("rows,cols", [(1, 64), (33, 1000), (5, 1001)])
def test_a_32_bit_stream_that_begins_with_the_block(block, mode, rows, cols):
    """Without x the type of h is asked for: not rounded to the block's 16 bits."""
    c = Case(rows, cols, F32, block, *mode, residual=False)
    h, y, stats = fo.fused_block_norm(None, c.f, stats=True, stream_type=F32, **c.how())
    want = ref.block_norm(None, host(c.f), **c.host_how())
    assert h.dtype == F32 and (y is None or y.dtype == block)
    close(h, *want["h"], unit(F32), "h")
    if c.pre:
        close(y, *want["y"], unit(F32), "y")
    c.check_backward(h, stats)
    out = torch.empty(rows, cols, device="cuda")
    again, _, _ = fo.fused_block_norm(None, c.f, out_h=out, stream_type=F32, **c.how())
    assert again is out and torch.equal(out, h)


def test_stream_types_that_are_refused():
    x, f = torch.zeros(3, 8, device="cuda"), torch.zeros(3, 8, dtype=BF16, device="cuda")
    h, _, _ = fo.fused_block_norm(x, f, stream_type=F32)
    assert h.dtype == F32
    for kw in (dict(x=x, f=f, stream_type=BF16), dict(f=f, stream_type=F16), dict(f=f, stream_type=F64), dict(f=f, stream_type="float32"),
               dict(f=f, out_h=x, stream_type=BF16)):
        with pytest.raises(ValueError):
            fo.fused_block_norm(**kw)


@pytest.mark.parametrize("vec", [BF16, F16, F32])
def test_no_gradient_of_y_for_the_norm_of_a_32_bit_stream(vec):
    """What the forward call takes the gradient takes too: 16-bit weights of a float32 stream, y not used further."""
    x = torch.randn(5, 64, device="cuda")
    pre = ("layer", torch.ones(64, dtype=vec, device="cuda"), torch.ones(64, dtype=vec, device="cuda"), 1e-6)
    h, y, stats = fo.fused_block_norm(x, pre=pre, stats=True)
    got = fo.fused_block_norm_grad(torch.ones_like(x), None, h, None, stats, pre=pre)
    assert y.dtype == vec and bool((got["x"] == 1).all()) and bool((got["pre_w"] == 0).all()) and bool((got["pre_b"] == 0).all())
