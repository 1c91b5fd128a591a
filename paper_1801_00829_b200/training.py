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


# The current stream's handle as a number, without a Stream object around it where this torch has that call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _index(t):
    """Number of the GPU that a tensor is on."""
    index = t.get_device()
    _require(index >= 0, "fused operators need CUDA tensors (no CPU path)")
    return index


def _call(name, index, *args):
    """Calls a C entry on the current stream of GPU `index`, which is made current if another one is."""
    fn = getattr(load_library(), name)
    if index == torch.cuda.current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status:
        _check(status, name)


_scratch = {}


def _workspace(index, nbytes):
    """(address, size) of the current stream's scratch (binding.workspace), looked up by numbers."""
    key = (index, _raw_stream(index))
    buf = _scratch.get(key)
    if buf is None or buf.numel() < nbytes:
        buf = _scratch[key] = workspace(torch.device("cuda", index), nbytes)
    return buf.data_ptr(), buf.numel()


def _matrix(t, shape, dtype, index, name):
    """(address, leading dimension) of a matrix of the call, zeros for None."""
    if t is None:
        return 0, 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise ValueError("%s: a %s matrix of %s on GPU %d is needed, not %s of %s on %s"
                         % (name, dtype, tuple(shape), index, t.dtype, tuple(t.shape), t.device))
    ld, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise ValueError("rows of %s must be contiguous" % name)
    if ld < shape[1]:
        if shape[0] > 1:
            raise ValueError("rows of %s overlap" % name)
        ld = shape[1]
    return t.data_ptr(), ld


def _vector(t, n, dtype, index, name):
    """Address of a contiguous vector of the call, 0 for None."""
    if t is None:
        return 0
    if t.shape != (n,) or t.dtype is not dtype or t.get_device() != index or not (n <= 1 or t.is_contiguous()):
        raise ValueError("%s: a contiguous %s vector of %d on GPU %d is needed, not %s of %s on %s"
                         % (name, dtype, n, index, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _norm(spec, cols, dtype, index, name):
    if spec is None:
        return _NO_NORM
    kind, weight, bias, eps = spec
    _require(kind in NORM_KIND, "norm kind %r" % (kind,))
    return NORM_KIND[kind], 0, eps, _vector(weight, cols, dtype, index, name), _vector(bias, cols, dtype, index, name)


def _gate(spec, shape, dtype, index):
    """(access, activation, address, leading dimension or stride)"""
    if spec is None:
        return 0, 0, 0, 0
    access, t, act = spec
    _require(access in ACCESS and act in ACTIVATION, "gate %r, activation %r" % (access, act))
    if access == "cell":
        ptr, ld = _matrix(t, shape, dtype, index, "gate")
    else:
        n = shape[0] if access == "row" else shape[1]
        if t.dim() == 2 and 1 in t.shape:                    # a column or row vector
            t = t[:, 0] if t.shape[1] == 1 and access == "row" else t[0]
        _require(t.shape == (n,) and t.dtype is dtype and t.get_device() == index, "gate is not a vector of %d %s"
                 % (n, dtype))
        ld = t.stride(0) if n > 1 else 1
        _require(ld >= 1 if access == "row" else ld == 1, "stride of the gate")
        ptr = t.data_ptr()
    return ACCESS[access], ACTIVATION[act], ptr, ld


def _types(stream, block, post, pre, col_scale):
    """Type codes of stream, block and vectors, and the vectors' type: that of the first one, or the block's."""
    vec = None if col_scale is None else col_scale.dtype
    for spec in (post, pre):
        if spec is not None and vec is None:
            vec = spec[1].dtype if spec[1] is not None else spec[2].dtype if spec[2] is not None else None
    vec = block if vec is None else vec
    if (stream, block) not in PAIRS:
        raise ValueError("no kernel for a %s stream and a %s block" % (stream, block))
    if vec is not block and not (vec is torch.float32 and block.itemsize == 2):
        raise ValueError("vectors of %s with a block of %s" % (vec, block))
    return (DTYPES[stream], DTYPES[block], DTYPES[vec]), vec


def _sum_type(block):
    return torch.float64 if block is torch.float64 else torch.float32


def _new(like, shape, dtype):
    """An uninitialised packed tensor on the GPU of `like`."""
    if like.dtype is dtype and like.shape == shape and like.is_contiguous():
        return torch.empty_like(like)                        # the shorter way
    return torch.empty(shape, dtype=dtype, device=like.device)


def fused_block_norm(x=None, f=None, post=None, gate=None, scale=1.0, col_scale=None, pre=None, out_h=None, out_y=None,
                     stats=False, block_type=None):
    """h = x + scale * col_scale * act(gate) * norm(f; post),  y = norm(h; pre), row by row in one pass.

    x (the residual stream) or f (the block's output) may be None; without f the result is the norm of
    x alone.  Returns (h, y, stats): h is x itself without f, y is None without `pre`; stats (float, 4 x
    rows, with stats=True) is what fused_block_norm_grad needs.  y has the type of f, or without f
    `block_type` (default: that of x).  out_h may be x.  x None: h has the type of f or of out_h."""
    first = x if x is not None else f
    _require(first is not None, "x or f is needed")
    index, shape = _index(first), first.shape
    _require(len(shape) == 2, "matrices are 2-D")
    rows, cols = shape
    stream = first.dtype if x is not None or out_h is None else out_h.dtype
    if f is not None:
        block = f.dtype
    else:
        block = block_type if block_type is not None else out_y.dtype if out_y is not None else stream
        _require(post is None and gate is None and col_scale is None, "post, gate and col_scale need a block output f")
    types, vec = _types(stream, block, post, pre, col_scale)
    xp, ldx = _matrix(x, shape, stream, index, "x")
    fp, ldf = _matrix(f, shape, block, index, "f")
    access, act, gp, ldg = _gate(gate, shape, block, index)
    post_s = _norm(post, cols, vec, index, "post")
    pre_s = _norm(pre, cols, vec, index, "pre")
    csp = _vector(col_scale, cols, vec, index, "col_scale")
    h, y, st, stp = out_h, out_y, None, 0
    if h is None and f is not None:
        h = _new(first, shape, stream)
    if y is None and pre is not None:
        y = _new(first if f is None else f, shape, block)
    _require(y is None or pre is not None, "out_y without a norm before the next block")
    if stats:
        st = torch.empty((4, rows), dtype=_sum_type(block), device=first.device)
        stp = st.data_ptr()
    hp, ldh = _matrix(h, shape, stream, index, "out_h")
    yp, ldy = _matrix(y, shape, block, index, "out_y")
    if hp or yp or stp:
        _call("fused_block_norm", index,
              _BLOCK_NORM.pack(rows, cols, *types, access, act, 0, xp, fp, gp, csp, ldx, ldf, ldg, scale, *post_s, *pre_s,
                               hp, yp, stp, ldh, ldy))
    return (x if h is None else h), y, st


def fused_block_norm_grad(dh=None, dy=None, h=None, f=None, stats=None, post=None, gate=None, scale=1.0, col_scale=None,
                          pre=None, residual=True):
    """Gradients of fused_block_norm from dh and dy, the gradients of its results (None: zero).

    h and stats come from the forward call; the rest are its arguments.  Returns a dict with "x" (with
    residual), and for each argument that was given "f", "gate", "col_scale", "post_w", "post_b", "pre_w",
    "pre_b".  Gradients of vectors, and of a gate per row or column, are float (double for float64)."""
    first = dh if dh is not None else dy
    _require(first is not None, "dh or dy is needed")
    index, shape = _index(first), first.shape
    _require(len(shape) == 2, "matrices are 2-D")
    rows, cols = shape
    if dy is not None:
        _require(pre is not None and h is not None, "dy needs `pre` and h")
    elif f is not None:
        pre = None                                           # nothing reaches the norm of h
    stream = dh.dtype if dh is not None else h.dtype
    block = f.dtype if f is not None else dy.dtype if dy is not None else stream
    _require(f is not None or (post is None and gate is None and col_scale is None),
             "post, gate and col_scale need a block output f")
    types, vec = _types(stream, block, post, pre, col_scale)
    dhp, lddh = _matrix(dh, shape, stream, index, "dh")
    dyp, lddy = _matrix(dy, shape, block, index, "dy")
    hp, ldh = _matrix(h if dy is not None else None, shape, stream, index, "h")
    fp, ldf = _matrix(f, shape, block, index, "f")
    access, act, gp, ldg = _gate(gate, shape, block, index)
    post_s = _norm(post, cols, vec, index, "post")
    pre_s = _norm(pre, cols, vec, index, "pre")
    csp = _vector(col_scale, cols, vec, index, "col_scale")
    sums, stp = _sum_type(block), 0
    if stats is not None:
        _require(stats.shape == (4, rows) and stats.dtype is sums and stats.is_contiguous() and stats.get_device() == index,
                 "stats is not 4 x %d of %s" % (rows, sums))
        stp = stats.data_ptr()

    # the vectors' gradients lie in one buffer
    names = [] if col_scale is None else ["col_scale"]
    for part, spec in (("post", post), ("pre", pre)):
        if spec is not None:
            names += [part + end for end, t in (("_w", spec[1]), ("_b", spec[2])) if t is not None]
    got, at = {}, {}
    dxp = dfp = dgp = 0
    if residual or f is None:
        got["x"] = dx = _new(first, shape, stream)
        dxp = dx.data_ptr()
    if f is not None:
        got["f"] = df = _new(f, shape, block)
        dfp = df.data_ptr()
    if gate is not None:
        got["gate"] = dg = _new(gate[1], gate[1].shape, block if gate[0] == "cell" else sums)
        dgp = dg.data_ptr()
    if names:
        flat = torch.empty((len(names), cols), dtype=sums, device=first.device)
        base, line = flat.data_ptr(), cols * sums.itemsize
        got.update(zip(names, flat.unbind(0)))
        at = {name: base + k * line for k, name in enumerate(names)}
    packed = _BLOCK_NORM_GRAD.pack(rows, cols, *types, access, act, 0, dhp, dyp, hp, fp, gp, csp, stp, lddh, lddy, ldh, ldf,
                                   ldg, scale, *post_s, *pre_s, dxp, dfp, dgp, cols, cols, cols, at.get("col_scale", 0),
                                   at.get("post_w", 0), at.get("post_b", 0), at.get("pre_w", 0), at.get("pre_b", 0))
    need = load_library().fused_block_norm_grad_workspace_bytes(rows, cols, types[1])
    _call("fused_block_norm_grad", index, packed, *_workspace(index, need))
    return got


# ------------------------------------------------------------------ many tensors
def _same(tensors, name, dtype=None, device=None):
    """The type and device that the tensors of a list share; contiguous, all of them."""
    if tensors:
        _index(tensors[0])
        dtype = tensors[0].dtype if dtype is None else dtype
        device = tensors[0].device if device is None else device
    for t in tensors:
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
        self.types = DTYPES.get(self.dtype, 1), DTYPES.get(self.out_dtype, 1)

    def __len__(self):
        return len(self.grads)


def tensor_list(grads, outs=None):
    """A TensorList of gradients; outs None: clipped in place."""
    return TensorList(grads, outs)


def _grad_call(name, grads, kind, max_norm, eps, result_type, device, types):
    grads = grads if isinstance(grads, TensorList) else TensorList(grads)
    _require(result_type in (torch.float32, torch.float64), "results are float32 or float64")
    _require(kind in GRAD_NORM_KIND, "norm kind %r" % (kind,))
    if grads.device is not None:
        device = grads.device
    elif device is None:                                     # an empty list
        device = torch.device("cuda", torch.cuda.current_device())
    result = torch.empty(2, dtype=result_type, device=device)
    index = result.get_device()
    ws = _workspace(index, load_library().fused_grad_workspace_bytes())
    _call(name, index, grads.packed, len(grads.grads), *grads.types[:types], GRAD_NORM_KIND[kind], max_norm, eps,
          result.data_ptr(), DTYPES[result_type], *ws)
    return result


def fused_grad_norm(grads, max_norm, kind="l2", eps=1e-6, result_type=torch.float32, device=None):
    """(norm, factor) of all gradients together, as a tensor of two on the device: the "l2" or "max" norm and
    min(1, max_norm / (norm + eps)).  grads: a TensorList or a list of tensors; device: for an empty list."""
    return _grad_call("fused_grad_norm", grads, kind, max_norm, eps, result_type, device, 1)


def fused_grad_clip(grads, max_norm, kind="l2", eps=1e-6, result_type=torch.float32, device=None):
    """fused_grad_norm, and every gradient times the factor into the list's outs (or in place)."""
    return _grad_call("fused_grad_clip", grads, kind, max_norm, eps, result_type, device, 2)


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
        self.types = DTYPES.get(self.dtype, 1), DTYPES.get(self.weight_dtype, 0)

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
    kind, at = 0, 0
    if factor is not None:
        _require(factor.numel() == 1 and factor.device == tensors.device and factor.dtype in (torch.float32, torch.float64),
                 "factor is not one float on the gradients' device")
        kind, at = DTYPES[factor.dtype], factor.data_ptr()
    _call("fused_adamw", tensors.device.index, tensors.packed, len(tensors.grads), *tensors.types, lr, betas[0], betas[1],
          eps, step, at, kind)
