"""Operators of a language model's step between the block norms (include/fusedops_lm.h): norms of queries and keys with the
position rotation, a gated linear recurrence, and the distillation loss.  Documentation and marshalling only; the calls are in the CPython
extension (csrc/lm_py.cpp).

Norms are given as for fused_block_norm, ``(kind, weight, bias, eps)`` with kind "rms" or "layer".  The calls record nothing for
autograd: they refuse tensors that require a gradient while gradients are recorded, and are meant for an autograd.Function or for
training code that goes backwards itself.  Arithmetic, states and sums are in 32 bits (64 for float64).
"""
from __future__ import annotations

from . import training as _training


def _native():
    return _training._extension or _training._native()


def fused_head_norm(q, k=None, q_norm=None, k_norm=None, rotate=None, out_q=None, out_k=None):
    """Norms of the heads' queries and keys and their rotation by position, in one pass: (q, k).

    q, k: (tokens, heads, dim) or (batch, tokens, heads, dim) with their own numbers of heads and any strides, dim <= 512; k may be
    None.  q_norm, k_norm: None, or a norm whose vectors are shared by the heads.
    rotate: None or (cos, sin, positions, pairing, sections): float32 tables (positions, pairs) (float64 beside float64) of cosines
    and sines; int32 or int64 positions of the tokens, (batch, tokens) or (tokens); "halves" (value j is turned with j + pairs) or "pairs"
    (2j with 2j + 1); the first 2 * pairs values of a head are turned.  sections: None, or for positions with several axes a tuple of
    their numbers of pairs (1 to 4, one section behind the other), with positions (axes, batch, tokens) or (axes, tokens).
    A position outside the tables gives NaN.  out_q may be q, and out_k k."""
    return _native().head_norm(q, k, q_norm, k_norm, rotate, out_q, out_k)


def fused_head_norm_grad(dq=None, dk=None, q=None, k=None, q_norm=None, k_norm=None, rotate=None, out_q=None, out_k=None):
    """Gradients of fused_head_norm from dq and dk, the gradients of its results (None: not wanted), and its arguments.

    Returns a dict with "q" and "k" (out_q and out_k where given; they may be dq and dk) and for each vector that was given "q_w", "q_b",
    "k_w", "k_b", float (double for float64).  q and k are needed where they have a norm."""
    return _native().head_norm_grad(dq, dk, q, k, q_norm, k_norm, rotate, out_q, out_k)


def fused_scan(x, gate, decay="sigmoid", mix="rest", state=None, reset=None, lengths=None, out=None, out_state=None):
    """h_t = a_t h_{t-1} + m(a_t) x_t for every channel, over the tokens: (h, last state).

    x, gate: (batch, tokens, channels) or (tokens, channels), channels neighbours in memory; the gate of x's type, or float32 beside 16
    bits.  decay: a is the gate itself ("value"), its "sigmoid", or its "exp"; mix: m is 1 ("one"), 1 - a ("rest"), or
    sqrt(1 - a^2) ("root").  state: None, or float (batch, channels) (float64 beside float64), the h before the first token.
    reset: None, or bool or uint8 (batch, tokens): where it is set nothing of the past enters h.  lengths: None, or int32 or int64 (batch,): behind its
    end a sequence's inputs are not looked at and h is zero; the last state is that at the end.
    A decoding step is a call with one token and the state.  out may be x, out_state may be state."""
    return _native().scan(x, gate, decay, mix, state, reset, lengths, out, out_state)


def fused_scan_grad(dh, x, gate, h, decay="sigmoid", mix="rest", state=None, reset=None, lengths=None, dlast=None):
    """Gradients of fused_scan from dh and dlast, the gradients of its results (either may be None: zero), its arguments and h.

    Returns a dict with "x", "gate" and, with a state, "state".  Behind a sequence's end gradients are zero.  x may be None with
    mix "one"."""
    return _native().scan_grad(dh, x, gate, h, decay, mix, state, reset, lengths, dlast)


def fused_distill(logits, ids, values, tail=None, temperature=1.0, stats=False):
    """The distillation loss of every row from the teacher's top logits: (loss, stats or None).

    logits: (rows, vocab); ids, values: (rows, entries), int32 or int64 and the logits' type (or float32 beside 16 bits): the
    teacher's entries and their logits, at most 1024; an entry with a negative id is none.
    tail None: the teacher's shares are the softmax of values / temperature over the entries, and the loss their divergence from the
    student's softmax(logits / temperature).  tail, float (rows,): the log-sum-exp of the teacher's whole row over temperature (zeros for values that
    are log probabilities, at temperature 1); the shares are exp(values / temperature - tail), and what is left of both
    distributions outside the entries is compared too.  One entry with the value 0 is the cross entropy.
    stats (float, 3 x rows, with stats=True) is what fused_distill_grad needs."""
    return _native().distill(logits, ids, values, tail, temperature, stats, False, None, None)


def fused_distill_grad(dloss, logits, ids, values, stats, tail=None, temperature=1.0, out=None):
    """The gradient of fused_distill's loss to the logits, times dloss, float (rows,) or None for ones.

    A row whose dloss is zero is not looked at, and its gradient is zero.  out may be the logits."""
    return _native().distill_grad(logits, ids, values, tail, temperature, dloss, stats, out)


def fused_distill_step(dloss, logits, ids, values, tail=None, temperature=1.0, out=None):
    """Loss and gradient in one pass over the logits, for a dloss that is known before: (loss, gradient).

    The loss is without dloss; it is zero where dloss is.  Otherwise as fused_distill and fused_distill_grad."""
    return _native().distill(logits, ids, values, tail, temperature, False, True, dloss, out)
