"""The training-step operators against plain float64 evaluations (oracle/training.py), at the sizes, types, layouts
and values where they can go wrong.

Tolerances.  A result is rounded once to its type (relative u, plus half the smallest subnormal); before that every
operation rounds to 32 bits (64 for float64).  A row's result passes through a sum, a reciprocal root and about a
dozen products, an activation among them (a few 2^-22): within 64 rounding units of the magnitude it was added
up from.  A column sum over n rows adds at most n of them more.
"""
import numpy as np
import pytest
import torch

import paper_1801_00829_b200 as fo
from oracle import training as ref

pytestmark = pytest.mark.gpu

F64, F32, BF16, F16 = torch.float64, torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F64, F64), (F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)]
ROUND = {F64: (2.0 ** -53, 0.0), F32: (2.0 ** -24, 2.0 ** -150), BF16: (2.0 ** -8, 2.0 ** -134), F16: (2.0 ** -11, 2.0 ** -25)}


def unit(block):
    return 2.0 ** -53 if block == F64 else 2.0 ** -24


def host(t):
    return None if t is None else t.detach().to(torch.float64).cpu().numpy()


def close(got, want, scale, u, what, rows=0):
    rel, least = ROUND[got.dtype]
    g = host(got)
    assert g.shape == want.shape, "%s: shape %s, not %s" % (what, g.shape, want.shape)
    limit = rel * np.abs(want) + least + (64 + rows) * u * scale
    bad = ~(np.abs(g - want) <= limit)
    assert not bad.any(), "%s: %d of %d off, first %r for %r (limit %r)" % (
        what, bad.sum(), bad.size, g[bad].flat[0], want[bad].flat[0], limit[bad].flat[0])


class Case:
    """Inputs of a block norm on the device and, as float64, on the host."""

    def __init__(self, rows, cols, stream, block, post, gate, act, pre, bias=False, wide=False, residual=True, block_out=True,
                 col_scale=True, pad=0, shift=0, seed=0):
        rng = np.random.RandomState(seed + rows * 7 + cols)
        vec = F32 if wide and block in (BF16, F16) else block

        def matrix(dtype, spread, mean=0.0):
            full = torch.from_numpy(rng.randn(rows, cols + pad) * spread + mean).to(dtype).cuda()
            if shift:                                       # rows that begin off a 16-byte boundary
                flat = torch.zeros(full.numel() + shift, dtype=dtype, device="cuda")
                flat[shift:] = full.reshape(-1)
                full = flat[shift:].reshape(rows, cols + pad)
            return full[:, :cols]

        def vector(n, dtype, spread=0.3, mean=0.0):
            return torch.from_numpy(rng.randn(n) * spread + mean).to(dtype).cuda()

        self.rows, self.cols, self.block, self.stream = rows, cols, block, stream
        self.x = matrix(stream, 1.5, 0.4) if residual or not block_out else None
        self.f = matrix(block, 0.7, -0.2) if block_out else None
        spec = lambda kind: (kind, vector(cols, vec, 0.2, 1.0), vector(cols, vec) if bias else None, 1e-5) if kind else None  # noqa: E731
        self.post = spec(post) if block_out else None
        self.pre = spec(pre)
        self.gate = None
        if gate and block_out:
            g = matrix(block, 1.5) if gate == "cell" else vector(rows if gate == "row" else cols, block, 1.5)
            self.gate = (gate, g, act)
        self.col_scale = vector(cols, vec, 0.3, 0.6) if col_scale and block_out else None
        self.scale = 0.75
        self.dh, self.dy = matrix(stream, 0.5), matrix(block, 0.5) if pre else None

    def how(self):
        return dict(post=self.post, gate=self.gate, scale=self.scale, col_scale=self.col_scale, pre=self.pre)

    def host_how(self):
        spec = lambda s: None if s is None else (s[0], host(s[1]), host(s[2]), s[3])  # noqa: E731
        gate = None if self.gate is None else (self.gate[0], host(self.gate[1]), self.gate[2])
        return dict(post=spec(self.post), gate=gate, scale=self.scale, col_scale=host(self.col_scale), pre=spec(self.pre))

    def check_forward(self):
        h, y, stats = fo.fused_block_norm(self.x, self.f, stats=True, **self.how())
        want = ref.block_norm(host(self.x), host(self.f), **self.host_how())
        u = unit(self.block)
        if self.f is not None:
            assert h.dtype == (self.stream if self.x is not None else self.block)
            close(h, *want["h"], u, "h")
        if self.pre is not None:
            assert y.dtype == self.block
            close(y, *want["y"], u, "y")
        big = np.abs(want["stats"]) + np.abs(want["h"][0]).max() + 1.0
        close(stats, want["stats"], big, u, "stats")
        return h, stats

    def check_backward(self, h, stats, dh="given"):
        dh = self.dh if isinstance(dh, str) else dh
        got = fo.fused_block_norm_grad(dh, self.dy, h if self.pre else None, self.f, stats, **self.how())
        want = ref.block_norm_grad(host(dh), host(self.dy), host(h), host(self.f), host(stats), **self.host_how())
        u = unit(self.block)
        names = {"x"} | ({"f"} if self.f is not None else set()) | ({"gate"} if self.gate else set())
        names |= {"col_scale"} if self.col_scale is not None else set()
        for part, spec in (("post", self.post), ("pre", self.pre)):
            names |= {part + "_w"} if spec and spec[1] is not None else set()
            names |= {part + "_b"} if spec and spec[2] is not None else set()
        assert set(got) == names
        for name in sorted(names):
            value, size = want[name]
            summed = name not in ("x", "f") and not (name == "gate" and self.gate[0] == "cell")
            assert got[name].dtype == ((F64 if self.block == F64 else F32) if summed else
                                       self.stream if name == "x" else self.block)
            close(got[name], value.reshape(got[name].shape), size.reshape(value.shape).reshape(got[name].shape), u, name,
                  rows=max(self.rows, self.cols) if summed else 0)


WIDTHS = [1, 2, 7, 8, 63, 64, 65, 128, 200, 256, 511, 512, 520, 1000, 1024, 1025, 2048, 2056, 4096, 4099, 8192, 8200, 12345,
          16384, 16392, 20001, 32768]
MODES = [("rms", "cell", "sigmoid", "rms"), ("layer", "row", "silu", "layer"), ("rms", "col", "tanh", "layer"),
         ("layer", None, "linear", "rms"), (None, "cell", "silu", "rms"), (None, None, "linear", "layer"),
         ("rms", "row", "linear", None), ("layer", "cell", "tanh", None), (None, "col", "linear", "rms"),
         ("rms", "cell", "linear", "layer"), ("layer", "col", "sigmoid", "rms")]


@pytest.mark.parametrize("stream,block", PAIRS)
@pytest.mark.parametrize("cols", WIDTHS)
def test_widths(stream, block, cols):
    for k, rows in enumerate((1, 5, 37) if cols <= 4100 else (1, 3)):
        post, gate, act, pre = MODES[(cols + 3 * k + PAIRS.index((stream, block))) % len(MODES)]
        c = Case(rows, cols, stream, block, post, gate, act, pre, bias=k == 1, wide=k == 2)
        c.check_backward(*c.check_forward())


@pytest.mark.parametrize("stream,block", PAIRS)
@pytest.mark.parametrize("mode", range(len(MODES)))
@pytest.mark.parametrize("rows,cols", [(33, 96), (19, 1000)])
def test_modes(stream, block, mode, rows, cols):
    for bias, wide, residual in ((False, False, True), (True, True, False)):
        c = Case(rows, cols, stream if residual else block, block, *MODES[mode], bias=bias, wide=wide, residual=residual,
                 col_scale=not bias)
        c.check_backward(*c.check_forward())


@pytest.mark.parametrize("stream,block", PAIRS)
@pytest.mark.parametrize("rows,cols", [(1, 4096), (257, 128), (700, 72), (64, 1003), (3, 9000)])
def test_norm_of_the_stream_alone(stream, block, rows, cols):
    for kind, bias in (("rms", False), ("layer", True)):
        c = Case(rows, cols, stream, block, None, None, "linear", kind, bias=bias, block_out=False)
        h, y, stats = fo.fused_block_norm(c.x, pre=c.pre, block_type=block, stats=True)
        assert h is c.x
        want = ref.block_norm(host(c.x), None, **c.host_how())
        close(y, *want["y"], unit(block), "y")
        c.check_backward(c.x, stats)
        c.check_backward(c.x, stats, dh=None)


@pytest.mark.parametrize("pad,shift", [(0, 1), (8, 0), (3, 0), (24, 8), (5, 3)])
@pytest.mark.parametrize("stream,block", [(BF16, BF16), (F32, F16), (F64, F64)])
def test_strides_and_offsets(stream, block, pad, shift):
    for rows, cols in ((9, 257), (6, 1000), (3, 2048)):
        c = Case(rows, cols, stream, block, "rms", "cell", "silu", "layer", bias=True, pad=pad, shift=shift)
        c.check_backward(*c.check_forward())


@pytest.mark.parametrize("rows", [1000, 2500])
@pytest.mark.parametrize("cols", [40, 130, 300, 1500])
def test_more_rows_than_the_grid(rows, cols):
    c = Case(rows, cols, BF16, BF16, "layer", "col", "sigmoid", "rms", bias=True)
    c.check_backward(*c.check_forward())


def test_outputs_given_in_place_and_padded():
    c = Case(21, 520, F32, BF16, "rms", "cell", "sigmoid", "rms")
    h0, y0, _ = fo.fused_block_norm(c.x, c.f, **c.how())
    y = torch.full((21, 600), 7.0, dtype=BF16, device="cuda")
    x = c.x.clone()
    h1, y1, _ = fo.fused_block_norm(x, c.f, out_h=x, out_y=y[:, :520], **c.how())
    assert h1 is x and torch.equal(x, h0) and torch.equal(y1, y0)
    assert bool((y[:, 520:] == 7.0).all())


def test_a_column_vector_gate_with_a_stride():
    c = Case(30, 100, F32, F32, "rms", "row", "sigmoid", "rms")
    wide = torch.zeros(30, 4, device="cuda")
    wide[:, 1] = c.gate[1]
    h0, _, _ = fo.fused_block_norm(c.x, c.f, **c.how())
    h1, _, _ = fo.fused_block_norm(c.x, c.f, **{**c.how(), "gate": ("row", wide[:, 1], "sigmoid")})
    h2, _, _ = fo.fused_block_norm(c.x, c.f, **{**c.how(), "gate": ("row", c.gate[1][:, None], "sigmoid")})
    assert torch.equal(h0, h1) and torch.equal(h0, h2)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_zero_rows_constant_rows_and_large_means(kind):
    for cols in (100, 1000, 5000):
        x = torch.zeros(4, cols, device="cuda")
        x[1] = 3.0
        x[2] = 1e4 + torch.linspace(-1, 1, cols, device="cuda")
        x[3, cols // 2] = 2e4
        _, y, st = fo.fused_block_norm(x, pre=(kind, None, None, 1e-6), stats=True)
        want = ref.block_norm(host(x), None, None, None, 1.0, None, (kind, None, None, 1e-6))
        close(y, *want["y"], unit(F32), "y")
        assert bool(torch.isfinite(y).all()) and bool((y[0] == 0).all())


def test_nan_and_infinity_stay_in_their_row():
    for cols in (96, 1000, 3000):
        c = Case(12, cols, F32, F32, "rms", "cell", "sigmoid", "layer")
        h0, y0, _ = fo.fused_block_norm(c.x, c.f, **c.how())
        c.x[3, cols - 1] = float("inf")
        c.f[7, 0] = float("nan")
        h1, y1, _ = fo.fused_block_norm(c.x, c.f, **c.how())
        keep = [i for i in range(12) if i not in (3, 7)]
        assert torch.equal(h0[keep], h1[keep]) and torch.equal(y0[keep], y1[keep])
        assert bool(torch.isnan(y1[7]).all()) and bool(torch.isnan(h1[7]).all())
        assert bool(torch.isinf(h1[3, cols - 1])) and bool(torch.isnan(y1[3, cols - 1]))


def test_empty():
    for rows, cols in ((0, 64), (3, 0), (0, 0)):
        x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
        w = torch.ones(cols, dtype=BF16, device="cuda")
        h, y, st = fo.fused_block_norm(x, x, post=("rms", w, None, 1e-6), pre=("layer", w, w, 1e-6), stats=True)
        assert h.shape == y.shape == (rows, cols)
        got = fo.fused_block_norm_grad(h, y, h, x, st, post=("rms", w, None, 1e-6), pre=("layer", w, w, 1e-6))
        assert got["x"].shape == (rows, cols) and bool((got["pre_w"] == 0).all()) and bool((got["post_w"] == 0).all())


@pytest.mark.parametrize("stream,vec,out", [(F32, BF16, BF16), (F32, F16, F16), (F32, F32, F32), (BF16, F32, BF16), (F64, F64, F64)])
def test_type_of_the_norm_of_the_stream_alone(stream, vec, out):
    x, w = torch.randn(5, 64, device="cuda").to(stream), torch.ones(64, dtype=vec, device="cuda")
    _, y, _ = fo.fused_block_norm(x, pre=("rms", w, None, 1e-6))
    assert y.dtype == out
    want = ref.block_norm(host(x), None, None, None, 1.0, None, ("rms", host(w), None, 1e-6))
    close(y, *want["y"], unit(stream), "y")


def test_without_a_gradient_of_y_or_of_h():
    c = Case(19, 130, BF16, BF16, "rms", "cell", "silu", "layer", bias=True)
    h, stats = c.check_forward()
    c.check_backward(h, stats, dh=None)
    got = fo.fused_block_norm_grad(c.dh, None, h, c.f, stats, **c.how())
    want = ref.block_norm_grad(host(c.dh), None, host(h), host(c.f), host(stats), **c.host_how())
    assert torch.equal(got["x"], c.dh) and bool((got["pre_w"] == 0).all()) and bool((got["pre_b"] == 0).all())
    close(got["f"], *want["f"], unit(BF16), "f")
    close(got["post_w"], *want["post_w"], unit(BF16), "post_w", rows=19)


def test_the_same_bits_twice():
    c = Case(600, 1000, BF16, BF16, "layer", "col", "silu", "layer", bias=True)
    h, stats = c.check_forward()
    a = fo.fused_block_norm_grad(c.dh, c.dy, h, c.f, stats, **c.how())
    b = fo.fused_block_norm_grad(c.dh, c.dy, h, c.f, stats, **c.how())
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("gate", [None, "cell", "row", "col"])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), (None, "rms"), ("layer", None)])
def test_gradient_against_differences(gate, post, pre):
    """The gradient of sum(h dh + y dy) in float64 against central differences: step 1e-5 leaves about 1e-10 of
    truncation and 1e-10 of rounding on values near 1."""
    c = Case(4, 13, F64, F64, post, gate, "silu", pre, bias=True)

    def loss(name=None, at=None, by=0.0):
        """The loss with element `at` of one argument moved."""
        how = c.how()
        x, f = c.x.clone(), c.f.clone()
        move = {"x": x, "f": f}
        if c.gate:
            g = c.gate[1].clone()
            how["gate"] = (c.gate[0], g, c.gate[2])
            move["gate"] = g
        cs = c.col_scale.clone()
        how["col_scale"] = move["col_scale"] = cs
        for part in ("post", "pre"):
            if how[part]:
                w, b = how[part][1].clone(), how[part][2].clone()
                how[part] = (how[part][0], w, b, how[part][3])
                move[part + "_w"], move[part + "_b"] = w, b
        if name:
            move[name].view(-1)[at] += by
        h, y, _ = fo.fused_block_norm(x, f, **how)
        total = (h * c.dh).sum()
        return (total + (y * c.dy).sum() if y is not None else total).item()

    h, _, stats = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    got = fo.fused_block_norm_grad(c.dh, c.dy, h, c.f, stats, **c.how())
    rng = np.random.RandomState(3)
    for name, g in got.items():
        for at in rng.choice(g.numel(), min(6, g.numel()), replace=False):
            want = (loss(name, at, 1e-5) - loss(name, at, -1e-5)) / 2e-5
            assert abs(g.reshape(-1)[at].item() - want) <= 1e-6 * (1.0 + abs(want)), (name, at)


def test_on_a_stream_of_its_own():
    c = Case(300, 1000, BF16, BF16, "rms", "cell", "sigmoid", "rms")
    h0, y0, st0 = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
    g0 = fo.fused_block_norm_grad(c.dh, c.dy, h0, c.f, st0, **c.how())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h1, y1, st1 = fo.fused_block_norm(c.x, c.f, stats=True, **c.how())
        g1 = fo.fused_block_norm_grad(c.dh, c.dy, h1, c.f, st1, **c.how())
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(h0, h1) and torch.equal(y0, y1) and all(torch.equal(g0[k], g1[k]) for k in g0)


def test_offsets_beyond_32_bits():
    """2.2e9 elements: the last rows lie where a 32-bit offset would have wrapped."""
    rows, cols = 270000, 8192
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    x = torch.ones(rows, cols, dtype=BF16, device="cuda")
    tail = torch.randn(3, cols, device="cuda").to(BF16)
    x[-3:] = tail
    w = torch.ones(cols, dtype=BF16, device="cuda")
    _, y, stats = fo.fused_block_norm(x, pre=("rms", w, None, 1e-6), stats=True)
    want = ref.block_norm(host(tail), None, None, None, 1.0, None, ("rms", host(w), None, 1e-6))
    close(y[-3:], *want["y"], unit(BF16), "y")
    assert bool((y[:-3:1000] == 1).all())
    got = fo.fused_block_norm_grad(None, y, x, None, stats, pre=("rms", w, None, 1e-6))
    wide = ref.block_norm_grad(None, host(y[-3:]), host(tail), None, host(stats[:, -3:]), None, None, 1.0, None,
                               ("rms", host(w), None, 1e-6))
    close(got["x"][-3:], *wide["x"], unit(BF16), "x")


def test_a_tensor_of_more_than_32_bits():
    n = (1 << 31) + 12345
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[-1], g[1 << 31], g[5] = 3.0, 4.0, 12.0
    norm, factor = host(fo.fused_grad_clip([g], 6.5, eps=0.0))
    assert norm == 13.0 and factor == 0.5
    assert g[-1].item() == 1.5 and g[1 << 31].item() == 2.0 and g[5].item() == 6.0


# ------------------------------------------------------------------ many tensors
SIZES = {"one": [1], "tiny": [1, 0, 3, 7, 8, 9, 15, 16, 17, 31, 0], "tile": [8191, 8192, 8193, 16384, 5],
         "ragged": [100003, 64, 1, 33333, 7, 250000, 4097], "forty": [777] * 40, "many": [50 + 13 * (k % 29) for k in range(1100)]}


def views(sizes, dtype, rng, spread, shift=0, packed=False):
    """Tensors of their own, or views into one buffer, tensor behind tensor."""
    total = sum(sizes)
    flat = torch.from_numpy(rng.randn(total + shift) * spread).to(dtype).cuda()[shift:]
    parts = list(torch.split(flat, sizes))
    return parts if packed else [p.clone() for p in parts]


@pytest.mark.parametrize("name", sorted(SIZES))
@pytest.mark.parametrize("gt,ot", [(F64, F64), (F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)])
@pytest.mark.parametrize("kind", ["l2", "max"])
def test_clip(name, gt, ot, kind):
    rng = np.random.RandomState(5)
    sizes = SIZES[name]
    for packed_in, shift in ((False, 0), (True, 1)):
        grads = views(sizes, gt, rng, 0.5, shift, packed_in)
        outs = views(sizes, ot, rng, 1.0, 3, True)
        want_norm, want_factor = ref.grad_norm([host(g) for g in grads], kind, 0.75, 1e-6)
        rt = F64 if gt == F64 else F32
        # sums of squares: 32 values in 32 bits, the rest in 64
        tol = 1e-13 if gt == F64 else 48 * 2.0 ** -24
        result = fo.fused_grad_clip(fo.tensor_list(grads, outs), 0.75, kind=kind, result_type=rt)
        norm, factor = host(result)
        assert abs(norm - want_norm) <= tol * want_norm and abs(factor - want_factor) <= tol * want_factor
        only = host(fo.fused_grad_norm(grads, 0.75, kind=kind, result_type=rt))
        assert only[0] == norm and only[1] == factor
        rel, least = ROUND[ot]
        for g, o in zip(grads, outs):
            want = host(g) * want_factor
            assert np.all(np.abs(host(o) - want) <= (rel + 2 * tol) * np.abs(want) + least)
        # in place
        fo.fused_grad_clip(grads, 0.75, kind=kind)
        if gt == ot:
            assert all(torch.equal(g, o) for g, o in zip(grads, outs)) or gt == F64


def test_nothing_beside_the_tensors_is_written():
    for ot in (F32, BF16):
        flat = torch.full((5000,), 9.0, dtype=ot, device="cuda")
        outs = [flat[7:1030], flat[1031:1034], flat[2000:4999]]
        grads = [torch.ones(o.numel(), dtype=BF16, device="cuda") for o in outs]
        fo.fused_grad_clip(fo.tensor_list(grads, outs), 0.001)
        keep = torch.ones(5000, dtype=torch.bool, device="cuda")
        for lo, hi in ((7, 1030), (1031, 1034), (2000, 4999)):
            keep[lo:hi] = False
        assert bool((flat[keep] == 9.0).all()) and bool((flat[~keep] != 9.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [1e-30, 1e-22, 1e-3, 1e15, 1e30])
def test_norms_near_the_ends_of_the_range(dtype, value):
    grads = [torch.full((n,), value, dtype=dtype, device="cuda") for n in (10000, 3, 517)]
    want, _ = ref.grad_norm([host(g) for g in grads], "l2", 1.0, 1e-6)
    norm = host(fo.fused_grad_norm(grads, 1.0, result_type=F64))[0]
    assert abs(norm - want) <= 48 * 2.0 ** -24 * want


@pytest.mark.parametrize("kind", ["l2", "max"])
def test_clip_with_nan_infinity_zero_and_nothing(kind):
    base = [torch.ones(n, device="cuda") for n in (9000, 5, 30000)]
    for spot in ((0, 0), (1, 4), (2, 29999)):
        g = [t.clone() for t in base]
        g[spot[0]][spot[1]] = float("nan")
        norm, factor = host(fo.fused_grad_clip(g, 1.0, kind=kind))
        assert np.isnan(norm) and np.isnan(factor) and bool(torch.isnan(g[2]).all())
        g = [t.clone() for t in base]
        g[spot[0]][spot[1]] = float("-inf")
        norm, factor = host(fo.fused_grad_clip(g, 1.0, kind=kind))
        assert norm == np.inf and factor == 0.0
        assert bool(torch.isnan(g[spot[0]][spot[1]])) and sum(int((t == 0).sum()) for t in g) == 39004
    zero = [torch.zeros(100, device="cuda")]
    assert host(fo.fused_grad_clip(zero, 1.0, kind=kind)).tolist() == [0.0, 1.0]
    assert host(fo.fused_grad_clip([], 1.0, kind=kind)).tolist() == [0.0, 1.0]
    assert host(fo.fused_grad_clip([torch.zeros(0, device="cuda")], 1.0, kind=kind)).tolist() == [0.0, 1.0]
    small = [t * 1e-3 for t in base]
    keep = [t.clone() for t in small]
    assert host(fo.fused_grad_clip(small, 1.0, kind=kind))[1] == 1.0 and all(torch.equal(a, b) for a, b in zip(small, keep))


@pytest.mark.parametrize("name", sorted(SIZES))
@pytest.mark.parametrize("gt,wt", [(F64, None), (F32, None), (BF16, BF16), (F16, F16), (F32, F16), (BF16, None)])
def test_adamw(name, gt, wt):
    rng = np.random.RandomState(11)
    sizes = SIZES[name]
    wide = F64 if gt == F64 else F32
    for packed, shift in ((True, 0), (True, 2), (False, 0)):
        p, m = (views(sizes, wide, rng, s, shift, packed) for s in (0.1, 0.01))
        v = [t.square() for t in views(sizes, wide, rng, 0.01, shift, packed)]
        g = views(sizes, gt, rng, 0.02, 0, False)
        outs = [views(sizes, wide, rng, 1.0, shift + k, True) for k in range(3)]
        w = views(sizes, wt, rng, 1.0, shift, packed) if wt else None
        decay = [0.1 if k % 2 else 0.0 for k in range(len(sizes))]
        factor = torch.tensor([0.4], dtype=wide, device="cuda")
        hyper = dict(lr=1e-2, betas=(0.9, 0.98), eps=1e-8, step=7)
        fo.fused_adamw(fo.adam_list(p, g, m, v, decay=decay, outs=outs, weights=w), factor=factor, **hyper)
        u = unit(gt)
        for k in range(0, len(sizes), 1 if len(sizes) < 50 else 97):
            want = ref.adamw(host(p[k]), host(g[k]), host(m[k]), host(v[k]), host(factor)[0], decay=decay[k], **hyper)
            sizes_of = (np.abs(host(p[k])) + 1e-2 * (1 + np.abs(want[0] - host(p[k])) / 1e-2),
                        np.abs(host(m[k])) + np.abs(host(g[k])), want[2])
            for o, value, size in zip(outs, want, sizes_of):
                close(o[k], value, size, u, "adamw")
            if w is not None:
                assert torch.equal(w[k], outs[0][k].to(wt))
        ip = fo.adam_list(p, g, m, v, decay=decay)
        fo.fused_adamw(ip, factor=factor, **hyper)
        assert all(torch.equal(a, b) for a, b in zip(p + m + v, outs[0] + outs[1] + outs[2]))


def test_adamw_without_a_factor_and_first_step():
    p, m, v = ([torch.zeros(5, device="cuda")] for _ in range(3))
    g = [torch.tensor([1.0, -2.0, 0.0, 1e-3, 5.0], device="cuda")]
    fo.fused_adamw(fo.adam_list(p, g, m, v), lr=0.1, step=1)
    # the first step moves every parameter by lr against its gradient's sign; 0 / eps stays
    assert np.allclose(host(p[0]), [-0.1, 0.1, 0.0, -0.1, -0.1], rtol=0, atol=2e-6)
    fo.fused_adamw(fo.adam_list([], [], [], []), lr=0.1)
