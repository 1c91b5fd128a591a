"""The training-step operators (include/fusedops_train.h): block norm and its gradient, gradient
clipping and AdamW over many tensors.  Argument checks and marshalling only, like binding.py.

Norms are given as ``(kind, weight, bias, eps)`` with kind "rms" or "layer" and weight / bias a vector
or None; a gate as ``(access, tensor, activation)`` with access "cell", "row" or "col" as for
side inputs, and activation "linear", "sigmoid", "silu" or "tanh".

The calls are made once per layer and step, on inputs that may be one token: the C structs are
packed by ``struct`` in one go rather than field by field.
"""
from __future__ import annotations

import struct

import torch

from .binding import ACCESS, _check, load_library, workspace

DTYPES = {torch.float64: 0, torch.float32: 1, torch.bfloat16: 2, torch.float16: 3}
PAIRS = {(s, s) for s in DTYPES} | {(torch.float32, torch.bfloat16), (torch.float32, torch.float16)}
NORM_KIND = {"rms": 1, "layer": 2}
ACTIVATION = {"linear": 0, "sigmoid": 1, "silu": 2, "tanh": 3}
GRAD_NORM_KIND = {"l2": 0, "max": 1}

_NORM = "iidQQ"
_BLOCK_NORM = struct.Struct("qq6i4Q3qd" + _NORM * 2 + "3Q2q")
_BLOCK_NORM_GRAD = struct.Struct("qq6i7Q5qd" + _NORM * 2 + "3Q3q5Q")
_NO_NORM = (0, 0, 0.0, 0, 0)


def _require(ok, text):
    if not ok:
        raise ValueError(text)


def _device(t):
    _require(t.device.type == "cuda", "fused operators need CUDA tensors (no CPU path)")
    return t.device


class _OnDevice:
    """Makes `device` current for a call if another one is."""

    def __init__(self, device):
        self.other = torch.cuda.device(device) if device.index != torch.cuda.current_device() else None

    def __enter__(self):
        if self.other is not None:
            self.other.__enter__()

    def __exit__(self, *error):
        if self.other is not None:
            self.other.__exit__(*error)


class _Rows:
    """Checks of one call's matrices and vectors: all rows x cols on one device, rows contiguous."""

    def __init__(self, like, cols_of):
        _require(cols_of.dim() == 2, "matrices are 2-D")
        self.rows, self.cols = cols_of.shape
        self.device = _device(like)
        self.vec_type = None

    def matrix(self, t, dtype, name):
        """(address, leading dimension) of a matrix of the call."""
        if t is None:
            return 0, 0
        _require(t.shape == (self.rows, self.cols), "%s is not %d x %d" % (name, self.rows, self.cols))
        _require(t.dtype == dtype, "%s is %s, not %s" % (name, t.dtype, dtype))
        _require(t.device == self.device, "%s is on another device" % name)
        ld, inner = t.stride()
        _require(inner == 1 or self.cols <= 1, "rows of %s must be contiguous" % name)
        if ld < self.cols:
            _require(self.rows <= 1, "rows of %s overlap" % name)
            ld = self.cols
        return t.data_ptr(), ld

    def vector(self, t, name):
        """Address of a vector over the columns; all of a call have one type."""
        if t is None:
            return 0
        _require(t.shape == (self.cols,) and (self.cols <= 1 or t.stride(0) == 1), "%s is not a contiguous vector of %d"
                 % (name, self.cols))
        _require(t.device == self.device, "%s is on another device" % name)
        if self.vec_type is None:
            self.vec_type = t.dtype
        _require(t.dtype == self.vec_type, "weights, biases and col_scale have different types")
        return t.data_ptr()

    def norm(self, spec, name):
        if spec is None:
            return _NO_NORM
        kind, weight, bias, eps = spec
        _require(kind in NORM_KIND, "norm kind %r" % (kind,))
        return NORM_KIND[kind], 0, float(eps), self.vector(weight, name + " weight"), self.vector(bias, name + " bias")

    def gate(self, spec, dtype):
        """(access, activation, address, leading dimension or stride)"""
        if spec is None:
            return 0, 0, 0, 0
        access, t, act = spec
        _require(access in ACCESS and act in ACTIVATION, "gate %r, activation %r" % (access, act))
        if access == "cell":
            ptr, ld = self.matrix(t, dtype, "gate")
        else:
            n = self.rows if access == "row" else self.cols
            t = t.reshape(-1) if t.dim() == 2 and t.is_contiguous() else t
            _require(t.shape == (n,) and t.dtype == dtype and t.device == self.device, "gate is not a vector of %d %s"
                     % (n, dtype))
            ld = t.stride(0) if n > 1 else 1
            _require(ld >= 1 if access == "row" else ld == 1, "stride of the gate")
            ptr = t.data_ptr()
        return ACCESS[access], ACTIVATION[act], ptr, ld

    def types(self, stream, block):
        """(stream, block, vector) type codes; without vectors the block's type stands for theirs."""
        _require((stream, block) in PAIRS, "no kernel for a %s stream and a %s block" % (stream, block))
        vec = block if self.vec_type is None else self.vec_type
        _require(vec == block or (vec == torch.float32 and block.itemsize == 2), "vectors of %s with a block of %s"
                 % (vec, block))
        return DTYPES[stream], DTYPES[block], DTYPES[vec]


def _sum_type(block):
    return torch.float64 if block == torch.float64 else torch.float32


def fused_block_norm(x=None, f=None, post=None, gate=None, scale=1.0, col_scale=None, pre=None, out_h=None, out_y=None,
                     stats=False, block_type=None):
    """h = x + scale * col_scale * act(gate) * norm(f; post),  y = norm(h; pre), row by row in one pass.

    x (the residual stream) or f (the block's output) may be None; without f the result is the norm of
    x alone.  Returns (h, y, stats): h is x itself without f, y is None without `pre`; stats (float, 4 x
    rows, with stats=True) is what fused_block_norm_grad needs.  y has the type of f, or without f
    `block_type` (default: that of x).  out_h may be x.  x None: h has the type of f or of out_h."""
    _require(x is not None or f is not None, "x or f is needed")
    first = x if x is not None else f
    c = _Rows(first, first)
    if f is not None:
        block = f.dtype
        stream = x.dtype if x is not None else out_h.dtype if out_h is not None else block
    else:
        stream = x.dtype
        block = block_type if block_type is not None else out_y.dtype if out_y is not None else stream
        _require(post is None and gate is None and col_scale is None, "post, gate and col_scale need a block output f")
    xp, ldx = c.matrix(x, stream, "x")
    fp, ldf = c.matrix(f, block, "f")
    access, act, gp, ldg = c.gate(gate, block)
    post_s, pre_s, csp = c.norm(post, "post"), c.norm(pre, "pre"), c.vector(col_scale, "col_scale")
    types = c.types(stream, block)
    h = out_h
    if h is None and f is not None:
        h = torch.empty((c.rows, c.cols), dtype=stream, device=c.device)
    y = out_y
    if y is None and pre is not None:
        y = torch.empty((c.rows, c.cols), dtype=block, device=c.device)
    _require(y is None or pre is not None, "out_y without a norm before the next block")
    st = torch.empty((4, c.rows), dtype=_sum_type(block), device=c.device) if stats else None
    hp, ldh = c.matrix(h, stream, "out_h")
    yp, ldy = c.matrix(y, block, "out_y")
    if hp or yp or stats:
        packed = _BLOCK_NORM.pack(c.rows, c.cols, *types, access, act, 0, xp, fp, gp, csp, ldx, ldf, ldg, scale, *post_s,
                                  *pre_s, hp, yp, st.data_ptr() if stats else 0, ldh, ldy)
        with _OnDevice(c.device):
            _check(load_library().fused_block_norm(packed, torch.cuda.current_stream(c.device).cuda_stream),
                   "fused_block_norm")
    return (x if f is None and h is None else h), y, st


def fused_block_norm_grad(dh=None, dy=None, h=None, f=None, stats=None, post=None, gate=None, scale=1.0, col_scale=None,
                          pre=None, residual=True):
    """Gradients of fused_block_norm from dh and dy, the gradients of its results (None: zero).

    h and stats come from the forward call; the rest are its arguments.  Returns a dict with "x" (with
    residual), and for each argument that was given "f", "gate", "col_scale", "post_w", "post_b", "pre_w",
    "pre_b".  Gradients of vectors, and of a gate per row or column, are float (double for float64)."""
    first = dh if dh is not None else dy
    _require(first is not None, "dh or dy is needed")
    c = _Rows(first, first)
    _require(dy is None or (pre is not None and h is not None), "dy needs `pre` and h")
    like_stream = dh if dh is not None else h
    like_block = f if f is not None else dy
    stream = like_stream.dtype
    block = like_block.dtype if like_block is not None else stream
    _require(f is not None or (post is None and gate is None and col_scale is None),
             "post, gate and col_scale need a block output f")
    if dy is None:
        pre = None if f is not None else pre
    dhp, lddh = c.matrix(dh, stream, "dh")
    dyp, lddy = c.matrix(dy, block, "dy")
    hp, ldh = c.matrix(h if dy is not None else None, stream, "h")
    fp, ldf = c.matrix(f, block, "f")
    access, act, gp, ldg = c.gate(gate, block)
    post_s, pre_s, csp = c.norm(post, "post"), c.norm(pre, "pre"), c.vector(col_scale, "col_scale")
    types = c.types(stream, block)
    sums = _sum_type(block)
    if stats is not None:
        _require(stats.shape == (4, c.rows) and stats.dtype == sums and stats.is_contiguous() and stats.device == c.device,
                 "stats is not 4 x %d of %s" % (c.rows, sums))
    got = {}

    def make(name, shape, dtype, wanted):
        if not wanted:
            return 0
        got[name] = t = torch.empty(shape, dtype=dtype, device=c.device)
        return t.data_ptr()

    cells, cols = (c.rows, c.cols), (c.cols,)
    dxp = make("x", cells, stream, residual or f is None)
    dfp = make("f", cells, block, f is not None)
    dgp = 0
    if gate is not None:
        dgp = make("gate", gate[1].shape, block if gate[0] == "cell" else sums, True)
    dcsp = make("col_scale", cols, sums, col_scale is not None)
    dpost, dpre = ([make(name + end, cols, sums, spec is not None and spec[at] is not None) for end, at in (("_w", 1), ("_b", 2))]
                   for name, spec in (("post", post), ("pre", pre)))
    packed = _BLOCK_NORM_GRAD.pack(c.rows, c.cols, *types, access, act, 0, dhp, dyp, hp, fp, gp, csp,
                                   stats.data_ptr() if stats is not None else 0, lddh, lddy, ldh, ldf, ldg, scale,
                                   *post_s, *pre_s, dxp, dfp, dgp, c.cols, c.cols, c.cols, dcsp, *dpost, *dpre)
    lib = load_library()
    with _OnDevice(c.device):
        need = lib.fused_block_norm_grad_workspace_bytes(c.rows, c.cols, types[1])
        ws = workspace(c.device, need)
        _check(lib.fused_block_norm_grad(packed, ws.data_ptr(), ws.numel(),
                                         torch.cuda.current_stream(c.device).cuda_stream), "fused_block_norm_grad")
    return got


# ------------------------------------------------------------------ many tensors
def _same(tensors, name, dtype=None, device=None):
    """The type and device that the tensors of a list share; contiguous, all of them."""
    for t in tensors:
        dtype = t.dtype if dtype is None else dtype
        device = _device(t) if device is None else device
        _require(t.dtype == dtype and t.device == device, "%s: tensors of one type on one device are needed" % name)
        _require(t.is_contiguous(), "%s: tensors must be contiguous" % name)
    return dtype, device


def _same_sizes(tensors, others, name):
    _require(len(tensors) == len(others), "%s: %d tensors for %d" % (name, len(others), len(tensors)))
    _require(all(a.numel() == b.numel() for a, b in zip(tensors, others)), "%s: sizes differ" % name)


class TensorList:
    """Gradients, and where their clipped values go: built once for buffers that a program keeps, or per call."""

    def __init__(self, grads, outs=None):
        self.grads = list(grads)
        self.outs = self.grads if outs is None else list(outs)
        self.dtype, self.device = _same(self.grads, "grads")
        _require(self.dtype is None or self.dtype in DTYPES, "no kernel for gradients of %s" % self.dtype)
        self.out_dtype = self.dtype
        if outs is not None:
            _same_sizes(self.grads, self.outs, "outs")
            self.out_dtype, _ = _same(self.outs, "outs", device=self.device)
            low = self.dtype in (torch.bfloat16, torch.float16)
            _require(self.out_dtype == self.dtype or (low and self.out_dtype == torch.float32),
                     "clipped values of %s from gradients of %s" % (self.out_dtype, self.dtype))
        flat = [v for g, o in zip(self.grads, self.outs) for v in (g.data_ptr(), o.data_ptr(), g.numel())]
        self.packed = struct.pack("QQq" * len(self.grads), *flat)

    def __len__(self):
        return len(self.grads)


def tensor_list(grads, outs=None):
    """A TensorList of gradients; outs None: clipped in place."""
    return TensorList(grads, outs)


def _grad_call(grads, result_type, device):
    grads = grads if isinstance(grads, TensorList) else TensorList(grads)
    device = grads.device or device or torch.device("cuda", torch.cuda.current_device())
    _require(result_type in (torch.float32, torch.float64), "results are float32 or float64")
    return grads, device, torch.empty(2, dtype=result_type, device=device)


def fused_grad_norm(grads, max_norm, kind="l2", eps=1e-6, result_type=torch.float32, device=None):
    """(norm, factor) of all gradients together, as a tensor of two on the device: the "l2" or "max" norm and
    min(1, max_norm / (norm + eps)).  grads: a TensorList or a list of tensors."""
    grads, device, result = _grad_call(grads, result_type, device)
    lib = load_library()
    with _OnDevice(device):
        ws = workspace(device, lib.fused_grad_workspace_bytes())
        _check(lib.fused_grad_norm(grads.packed, len(grads), DTYPES.get(grads.dtype, 1), GRAD_NORM_KIND[kind], max_norm,
                                   eps, result.data_ptr(), DTYPES[result_type], ws.data_ptr(), ws.numel(),
                                   torch.cuda.current_stream(device).cuda_stream), "fused_grad_norm")
    return result


def fused_grad_clip(grads, max_norm, kind="l2", eps=1e-6, result_type=torch.float32, device=None):
    """fused_grad_norm, and every gradient times the factor into the list's outs (or in place)."""
    grads, device, result = _grad_call(grads, result_type, device)
    lib = load_library()
    with _OnDevice(device):
        ws = workspace(device, lib.fused_grad_workspace_bytes())
        _check(lib.fused_grad_clip(grads.packed, len(grads), DTYPES.get(grads.dtype, 1), DTYPES.get(grads.out_dtype, 1),
                                   GRAD_NORM_KIND[kind], max_norm, eps, result.data_ptr(), DTYPES[result_type],
                                   ws.data_ptr(), ws.numel(), torch.cuda.current_stream(device).cuda_stream),
               "fused_grad_clip")
    return result


class AdamList:
    """Parameters, gradients and moments of one AdamW update, and where the new values go."""

    def __init__(self, params, grads, m, v, decay=0.0, outs=None, weights=None):
        self.params, self.grads, self.m, self.v = list(params), list(grads), list(m), list(v)
        self.outs = [list(o) for o in outs] if outs is not None else [self.params, self.m, self.v]
        self.weights = list(weights) if weights is not None else None
        self.dtype, self.device = _same(self.grads, "grads")
        _require(self.dtype is None or self.dtype in DTYPES, "no kernel for gradients of %s" % self.dtype)
        wide = torch.float64 if self.dtype == torch.float64 else torch.float32
        _require(len(self.outs) == 3, "outs are (params, m, v)")
        for name, ts in zip(("params", "m", "v", "params out", "m out", "v out"), [self.params, self.m, self.v] + self.outs):
            _same_sizes(self.grads, ts, name)
            _same(ts, name, wide, self.device)
        self.weight_dtype = None
        if self.weights is not None:
            _same_sizes(self.grads, self.weights, "weights")
            self.weight_dtype, _ = _same(self.weights, "weights", device=self.device)
            _require(self.weight_dtype in (None, torch.bfloat16, torch.float16), "weights are bfloat16 or float16")
        n = len(self.grads)
        decay = [float(decay)] * n if isinstance(decay, (int, float)) else [float(d) for d in decay]
        _require(len(decay) == n, "decay: %d values for %d tensors" % (len(decay), n))
        lists = [self.params, self.grads, self.m, self.v] + self.outs + ([self.weights] if self.weights is not None else [])
        none = [0] if self.weights is None else []
        flat = []
        for k in range(n):
            flat += [ts[k].data_ptr() for ts in lists] + none + [self.grads[k].numel(), decay[k]]
        self.packed = struct.pack("8Qqd" * n, *flat)

    def __len__(self):
        return len(self.grads)


def adam_list(params, grads, m, v, decay=0.0, outs=None, weights=None):
    """An AdamList.  outs: (params, m, v) of the new values, None: in place; weights: 16-bit copies of the new
    parameters; decay: one value, or one per tensor."""
    return AdamList(params, grads, m, v, decay, outs, weights)


def fused_adamw(tensors, lr, betas=(0.9, 0.999), eps=1e-8, step=1, factor=None):
    """One AdamW step over an AdamList.  factor: None, or a tensor of one value on the device that the
    gradients are multiplied by (result[1:2] of fused_grad_norm)."""
    if len(tensors) == 0:
        return
    device, kind = tensors.device, 0
    if factor is not None:
        _require(factor.numel() == 1 and factor.device == device and factor.dtype in (torch.float32, torch.float64),
                 "factor is not one float on the gradients' device")
        kind = DTYPES[factor.dtype]
    with _OnDevice(device):
        _check(load_library().fused_adamw(tensors.packed, len(tensors), DTYPES[tensors.dtype],
                                          DTYPES.get(tensors.weight_dtype, 0), lr, betas[0], betas[1], eps, step,
                                          factor.data_ptr() if factor is not None else 0, kind,
                                          torch.cuda.current_stream(device).cuda_stream), "fused_adamw")
