"""The training-step operators (include/fusedops_train.h): block norm and its gradient, gradient
clipping and AdamW over many tensors.  Argument checks and marshalling only, like binding.py; the calls
themselves are in a CPython extension (csrc/training_py.cpp).

Norms are given as ``(kind, weight, bias, eps)`` with kind "rms" or "layer" and weight / bias a vector
or None; a gate as ``(access, tensor, activation)`` with access "cell", "row" or "col" as for
side inputs, and activation "linear", "sigmoid", "silu" or "tanh".

The calls record nothing for autograd: fused_block_norm and its gradient refuse tensors that require a gradient while gradients
are recorded, and are meant for an autograd.Function or for training code that goes backwards itself.  Clipping and AdamW
write their tensors as an optimiser does.
"""
from __future__ import annotations

import importlib.util
import struct

import torch

from . import build as _build
from .binding import FusedOpsError, load_library, workspace

GRAD_NORM_KIND = {"l2": 0, "max": 1}


def _require(ok, text):
    if not ok:
        raise ValueError(text)


_extension = None


def _native():
    """The CPython extension, built if it is missing or stale."""
    global _extension
    if _extension is None:
        load_library()
        spec = importlib.util.spec_from_file_location(__package__ + "._training", _build.build_extension())
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.connect(FusedOpsError, lambda index, nbytes: workspace(torch.device("cuda", index), nbytes))
        _extension = module
    return _extension


def fused_block_norm(x=None, f=None, post=None, gate=None, scale=1.0, col_scale=None, pre=None, out_h=None, out_y=None,
                     stats=False, block_type=None, stream_type=None):
    """h = x + scale * col_scale * act(gate) * norm(f; post),  y = norm(h; pre), row by row in one pass.

    x (the residual stream) or f (the block's output) may be None; without f the result is the norm of
    x alone.  Returns (h, y, stats): h is x itself without f, y is None without `pre`; stats (float, 4 x
    rows, with stats=True) is what fused_block_norm_grad needs.  y has the type of f, or without f
    `block_type` (default: that of x; beside a float32 x that of the norm's weights).  out_h may be x.  x None: h has
    `stream_type` (float32 beside an f of 16 bits, where the stream begins with this block), or else the type of out_h or f."""
    return (_extension or _native()).block_norm(x, f, post, gate, scale, col_scale, pre, out_h, out_y, stats, block_type, stream_type)


def fused_block_norm_grad(dh=None, dy=None, h=None, f=None, stats=None, post=None, gate=None, scale=1.0, col_scale=None,
                          pre=None, residual=True):
    """Gradients of fused_block_norm from dh and dy, the gradients of its results (None: zero).

    h and stats come from the forward call; the rest are its arguments.  Returns a dict with "x" (with
    residual), and for each argument that was given "f", "gate", "col_scale", "post_w", "post_b", "pre_w",
    "pre_b".  Gradients of vectors, and of a gate per row or column, are float (double for float64)."""
    return (_extension or _native()).block_norm_grad(dh, dy, h, f, stats, post, gate, scale, col_scale, pre, residual)


# ------------------------------------------------------------------ many tensors
def _first(tensors, name):
    return getattr(tensors[0], name) if tensors else None


class TensorList:
    """Gradients, and where their clipped values go: built once for tensors that a program keeps, or per call.

    A list holds the tensors themselves.  Every call looks at them again, so a tensor may get other storage between two calls
    as long as type, device and size fit.  A program whose gradients are new tensors in every step (PyTorch's
    default after ``zero_grad``) needs a new list in every step: the old one still means the old gradients."""

    def __init__(self, grads, outs=None):
        self.grads = list(grads)
        self.outs = self.grads if outs is None else list(outs)
        (_extension or _native()).check_grads(self.grads, self.outs)

    dtype = property(lambda self: _first(self.grads, "dtype"))
    device = property(lambda self: _first(self.grads, "device"))
    out_dtype = property(lambda self: _first(self.outs, "dtype"))

    def __len__(self):
        return len(self.grads)


def tensor_list(grads, outs=None):
    """A TensorList of gradients; outs None: clipped in place."""
    return TensorList(grads, outs)


def _grad_call(grads, clip, kind, max_norm, eps, result_type, device):
    grads = grads if isinstance(grads, TensorList) else TensorList(grads)
    wide = result_type is torch.float64
    _require(wide or result_type is torch.float32, "results are float32 or float64")
    _require(kind in GRAD_NORM_KIND, "norm kind %r" % (kind,))
    index = -1
    if len(grads) == 0:
        device = torch.device("cuda" if device is None else device)
        _require(device.type == "cuda", "fused operators need CUDA tensors (no CPU path)")
        index = torch.cuda.current_device() if device.index is None else device.index
    return (_extension or _native()).grad_norm(grads.grads, grads.outs if clip else None, GRAD_NORM_KIND[kind], max_norm, eps,
                                               0 if wide else 1, index)


def fused_grad_norm(grads, max_norm, kind="l2", eps=1e-6, result_type=torch.float32, device=None):
    """(norm, factor) of all gradients together, as a tensor of two on the device: the "l2" or "max" norm and
    min(1, max_norm / (norm + eps)).  grads: a TensorList or a list of tensors; device: for an empty list."""
    return _grad_call(grads, False, kind, max_norm, eps, result_type, device)


def fused_grad_clip(grads, max_norm, kind="l2", eps=1e-6, result_type=torch.float32, device=None):
    """fused_grad_norm, and every gradient times the factor into the list's outs (or in place)."""
    return _grad_call(grads, True, kind, max_norm, eps, result_type, device)


class AdamList:
    """Parameters, gradients and moments of one AdamW update, and where the new values go.  What TensorList says of
    tensors that change holds here too."""

    def __init__(self, params, grads, m, v, decay=0.0, outs=None, weights=None):
        self.params, self.grads, self.m, self.v = list(params), list(grads), list(m), list(v)
        self.outs = [list(o) for o in outs] if outs is not None else [self.params, self.m, self.v]
        self.weights = list(weights) if weights is not None else None
        _require(len(self.outs) == 3, "outs are (params, m, v)")
        n = len(self.grads)
        decay = [float(decay)] * n if isinstance(decay, (int, float)) else [float(d) for d in decay]
        _require(len(decay) == n, "decay: %d values for %d tensors" % (len(decay), n))
        self._decay = struct.pack("%dd" % n, *decay)
        (_extension or _native()).check_adam(*self._lists())

    dtype = property(lambda self: _first(self.grads, "dtype"))
    device = property(lambda self: _first(self.grads, "device"))
    weight_dtype = property(lambda self: _first(self.weights or [], "dtype"))

    def _lists(self):
        return (self.params, self.grads, self.m, self.v, *self.outs, self.weights, self._decay)

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
    (_extension or _native()).adamw(*tensors._lists(), lr, betas[0], betas[1], eps, step, factor)
