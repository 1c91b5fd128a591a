"""Head norms with rotation, the gated recurrence and the distillation loss, step by step in float64.  Where a rounding error is
relative to more than the result itself, functions also return the magnitude a result was added up from (the same formula over
absolute values).
"""
import numpy as np


# ------------------------------------------------------------------------------------------------------------ head norms
def pair_places(pairs, pairing):
    """The two places of every pair."""
    j = np.arange(pairs)
    return (j, pairs + j) if pairing == "halves" else (2 * j, 2 * j + 1)


def angles(cos, sin, positions, sections):
    """cos and sin of every pair of every token, (batch, tokens, 1, pairs); NaN outside the tables.
    positions: (batch, tokens), or (axes, batch, tokens) with sections."""
    if sections is None:
        sections, positions = (cos.shape[1],), positions[None]
    at = np.repeat(np.arange(len(sections)), sections)
    rows = np.moveaxis(positions[at], 0, -1)
    ok = (rows >= 0) & (rows < cos.shape[0])
    rows = np.where(ok, rows, 0)
    j = np.arange(cos.shape[1])
    return tuple(np.where(ok, t[rows, j] if cos.shape[0] else np.nan, np.nan)[:, :, None] for t in (cos, sin))


def turn(t, size, pairing, c, s, back=False):
    if back:
        s = -s
    a, b = pair_places(c.shape[-1], pairing)
    out, osize = t.copy(), size.copy()
    out[..., a], out[..., b] = t[..., a] * c - t[..., b] * s, t[..., b] * c + t[..., a] * s
    for to in (a, b):
        osize[..., to] = size[..., a] * np.maximum(np.abs(c), np.abs(s)) + size[..., b] * np.maximum(np.abs(c), np.abs(s))
    return out, osize


def _normalised(x, kind, eps):
    mean = x.mean(-1, keepdims=True) if kind == "layer" else np.zeros(x.shape[:-1] + (1,))
    d = x - mean
    with np.errstate(divide="ignore"):
        r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return d * r, r, (np.abs(x) + np.abs(x).max(-1, keepdims=True, initial=0.0)) * r


def head_norm(x, norm, rotation):
    """(y, magnitude) of (batch, tokens, heads, dim); rotation: None or (c, s, pairing) with angles()."""
    y, size = x, np.abs(x)
    if norm is not None:
        kind, w, b, eps = norm
        n, _, size = _normalised(x, kind, eps)
        w = np.ones(x.shape[-1]) if w is None else w
        y, size = n * w, (size + np.abs(n)) * np.abs(w)
        if b is not None:
            y, size = y + b, size + np.abs(b)
    return (y, size) if rotation is None else turn(y, size, rotation[2], rotation[0], rotation[1])


def head_norm_grad(dy, x, norm, rotation):
    """{"x", "w", "b"}: (value, magnitude)."""
    g, gs = dy, np.abs(dy)
    if rotation is not None:
        g, gs = turn(g, gs, rotation[2], rotation[0], rotation[1], back=True)
    if norm is None:
        return {"x": (g, gs)}
    kind, w, _, eps = norm
    n, r, ns = _normalised(x, kind, eps)
    ns = ns + np.abs(n)
    w = np.ones(x.shape[-1]) if w is None else w
    a, size = g * w, gs * np.abs(w)
    back = a - n * (a * n).mean(-1, keepdims=True)
    bs = size + ns * (size * ns).mean(-1, keepdims=True)
    if kind == "layer":
        back, bs = back - a.mean(-1, keepdims=True), bs + size.mean(-1, keepdims=True)
    return {"x": (back * r, bs * r), "w": ((g * n).sum((0, 1, 2)), (gs * ns).sum((0, 1, 2))), "b": (g.sum((0, 1, 2)), gs.sum((0, 1, 2)))}


# ------------------------------------------------------------------------------------------------------------ recurrence
def decay(gate, kind):
    """a and 1 - a."""
    if kind == "value":
        return gate, 1.0 - gate
    if kind == "exp":
        return np.exp(gate), -np.expm1(gate)
    e = np.exp(-np.abs(gate))
    small = e / (1.0 + e)
    return np.where(gate >= 0, 1.0 / (1.0 + e), small), np.where(gate >= 0, small, 1.0 / (1.0 + e))


def decay_slope(a, rest, kind):
    return np.ones_like(a) if kind == "value" else a if kind == "exp" else a * rest


def mixed(a, rest, mix):
    with np.errstate(invalid="ignore"):
        return np.ones_like(a) if mix == "one" else rest if mix == "rest" else np.sqrt(rest * (1.0 + a))


def gate_error(gate, a, rest, kind):
    """By how many rounding units a may be off, and (relative) m(a).  The smaller of a and 1 - a is off by a few units of
    itself and the exponent's own, which grows with the gate; the larger by its rounding, a unit of 1."""
    own = 0.0 if kind == "value" else 24.0 + 4.0 * np.abs(gate)
    return (np.abs(a) + 1.0) * (0.0 if kind == "value" else 1.0) + np.minimum(np.abs(a), np.abs(rest)) * own, own + 8.0


def scan(x, gate, kind, mix, state, reset, lengths):
    """h, last and the bounds of their errors in rounding units of 32 (64) bits, before h is rounded to its type."""
    batch, tokens, channels = x.shape
    a, rest = decay(gate, kind)
    m = mixed(a, rest, mix)
    ea, em = gate_error(gate, a, rest, kind)
    em = np.broadcast_to(em, a.shape)
    h = np.zeros((batch, channels)) if state is None else state.copy()
    size, off = np.abs(h), np.zeros_like(h)
    out, outs, oute = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    for t in range(tokens):
        on = (t < lengths)[:, None]
        drop = reset[:, t, None]
        with np.errstate(invalid="ignore", over="ignore"):
            b = m[:, t] * x[:, t]
            new = np.where(drop, b, a[:, t] * h + b)
            ns = np.where(drop, np.abs(b), np.abs(a[:, t]) * size + np.abs(b))
            ne = np.where(drop, 0.0, np.abs(a[:, t]) * off + (ea[:, t] + 6.0 * np.abs(a[:, t])) * size) + (em[:, t] + 4.0) * np.abs(b) + 2.0 * ns
        h, size, off = np.where(on, new, h), np.where(on, ns, size), np.where(on, ne, off)
        out[:, t], oute[:, t] = np.where(on, h, 0.0), np.where(on, off, 0.0)
    return out, oute, h, off


def scan_grad(dh, x, gate, h, kind, mix, state, reset, lengths, dlast):
    """{"x", "gate", "state"}: (value, error in rounding units)."""
    batch, tokens, channels = gate.shape
    a, rest = decay(gate, kind)
    m = mixed(a, rest, mix)
    ea, em = gate_error(gate, a, rest, kind)
    em = np.broadcast_to(em, a.shape)
    da = decay_slope(a, rest, kind)
    with np.errstate(divide="ignore", invalid="ignore"):
        dm = np.zeros_like(a) if mix == "one" else -da if mix == "rest" else -a * da / m
    zero = np.zeros((batch, channels))
    x = np.zeros_like(gate) if x is None else x
    carry = zero.copy() if dlast is None else dlast.copy()
    size, off = np.abs(carry), zero.copy()
    got = {k: (np.zeros_like(gate), np.zeros_like(gate)) for k in ("x", "gate")}
    for t in reversed(range(tokens)):
        on, drop = (t < lengths)[:, None], reset[:, t, None]
        d = zero if dh is None else dh[:, t]
        before = np.where(drop, 0.0, h[:, t - 1] if t else zero if state is None else state)
        lam, ls = carry + d, size + np.abs(d)
        le = off + 2.0 * ls
        slope, ss = da[:, t] * before + dm[:, t] * x[:, t], np.abs(da[:, t] * before) + np.abs(dm[:, t] * x[:, t])
        for k, v, e in (("x", m[:, t] * lam, np.abs(m[:, t]) * (le + (em[:, t] + 4.0) * ls)),
                        ("gate", lam * slope, ss * (le + (2.0 * em[:, t] + 8.0) * ls))):
            got[k][0][:, t], got[k][1][:, t] = np.where(on, v, 0.0), np.where(on, e, 0.0)
        through, ts = np.where(drop, 0.0, a[:, t] * lam), np.where(drop, 0.0, np.abs(a[:, t]) * ls)
        te = np.where(drop, 0.0, np.abs(a[:, t]) * le + (ea[:, t] + 6.0 * np.abs(a[:, t])) * ls)
        carry, size, off = np.where(on, through, carry), np.where(on, ts, size), np.where(on, te, off)
    got["state"] = (carry, off)
    return got


# ------------------------------------------------------------------------------------------------------------ distillation
def distill(logits, ids, values, tail, temperature):
    """loss, stats (largest, sum, factor), gradient for dloss 1, and the student's probabilities.  One row after the other."""
    rows, vocab = logits.shape
    loss, stats, dz, q = np.zeros(rows), np.zeros((3, rows)), np.zeros_like(logits), np.zeros_like(logits)
    for r in range(rows):
        z, given = logits[r], ids[r] >= 0
        if (ids[r] >= vocab).any():
            loss[r], stats[2, r], dz[r] = np.nan, np.nan, np.nan
            continue
        at, v = ids[r][given], values[r][given] / temperature
        if tail is not None:
            p = np.exp(v - tail[r])
            rest = max(0.0, 1.0 - p.sum())
        else:
            p = np.exp(v - v.max()) / np.exp(v - v.max()).sum() if len(v) else v
            rest = 0.0
        with np.errstate(invalid="ignore", divide="ignore"):
            e = np.exp((z - z.max()) / temperature)
            total = e.sum()
            logq = (z - z.max()) / temperature - np.log(total)
            out = np.ones(vocab, dtype=bool)
            out[at] = False
            shares = np.bincount(at, weights=p, minlength=vocab)
            some = p > 0
            loss[r] = (p[some] * (np.log(p[some]) - logq[at][some])).sum()
            ratio = 0.0
            if e[out].sum() == 0 and rest <= 1 / 32:         # the rounding of values and tail
                rest = 0.0
            if rest > 0:
                ratio = rest / (e[out].sum() / total)
                loss[r] += rest * np.log(ratio)
            s = p.sum() + rest
            q[r] = e / total
            stats[:, r] = z.max(), total, s - ratio
            dz[r] = np.where(out, q[r] * (s - ratio), q[r] * s - shares) / temperature
    return loss, stats, dz, q
