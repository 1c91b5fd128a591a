"""The training-step operators, operator by operator in float64: block norm, its gradient, gradient
clipping, AdamW.  Every function also returns the magnitude each result was added up from
("scale": the same formula over absolute values), which is what a rounding error is relative to.
"""
import numpy as np


def activation(kind, g):
    """act(g) and act'(g)."""
    if kind == "linear":
        return g, np.ones_like(g)
    if kind == "tanh":
        t = np.tanh(g)
        return t, 1.0 - t * t
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-g))
    return (s, s * (1.0 - s)) if kind == "sigmoid" else (g * s, s * (1.0 + g * (1.0 - s)))


def statistics(t, kind, eps):
    """Mean (0 for "rms") and 1 / sqrt(mean((t - mean)^2) + eps) of every row."""
    mean = t.mean(axis=1) if kind == "layer" else np.zeros(t.shape[0])
    d = t - mean[:, None]
    with np.errstate(divide="ignore"):
        return mean, 1.0 / np.sqrt((d * d).mean(axis=1) + eps)


def _ones(v, cols):
    return np.ones(cols) if v is None else v


def _zeros(v, cols):
    return np.zeros(cols) if v is None else v


def norm(t, scale, spec):
    """norm(t), its statistics and its scale, from t and t's scale."""
    kind, weight, bias, eps = spec
    w, b = _ones(weight, t.shape[1]), _zeros(bias, t.shape[1])
    mean, r = statistics(t, kind, eps)
    out = (t - mean[:, None]) * r[:, None] * w + b
    # an error in a row's statistics reaches all of the row
    size = (scale + np.abs(t).max(axis=1, initial=0.0)[:, None]) * r[:, None] + 1.0
    return out, mean, r, size * np.abs(w) + np.abs(b)


def _gate(gate, rows):
    if gate is None:
        return None
    access, g, act = gate
    return access, (g.reshape(rows, 1) if access == "row" else g), act


def block_norm(x, f, post, gate, scale, col_scale, pre):
    """{"h", "y", "stats"}: (value, scale) of each; stats without a scale."""
    like = x if x is not None else f
    rows, cols = like.shape
    stats = np.zeros((4, rows))
    h = np.zeros((rows, cols)) if x is None else x
    size = np.abs(h)
    if f is not None:
        z, zs = f, np.abs(f)
        if post is not None:
            z, stats[0], stats[1], zs = norm(f, zs, post)
        if gate is not None:
            _, g, act = _gate(gate, rows)
            a, _ = activation(act, g)
            z, zs = z * a, zs * np.abs(a)
        k = scale * _ones(col_scale, cols)
        h, size = h + z * k, size + zs * np.abs(k)
    got = {"h": (h, size)}
    if pre is not None:
        y, stats[2], stats[3], ys = norm(h, size, pre)
        got["y"] = (y, ys)
    got["stats"] = stats
    return got


def _through(d, ds, t, stat, spec):
    """Gradient d (scale ds) of norm(t) -> of t, of the weight and of the bias."""
    kind, weight, bias, _ = spec
    w = _ones(weight, t.shape[1])
    mean, r = (s[:, None] for s in stat)
    n = (t - mean) * r
    ns = (np.abs(t) + np.abs(mean)) * r
    a, size = d * w, ds * np.abs(w)
    back = a - n * (a * n).mean(axis=1, keepdims=True)
    bs = size + ns * (size * ns).mean(axis=1, keepdims=True)
    if kind == "layer":
        back = back - a.mean(axis=1, keepdims=True)
        bs = bs + size.mean(axis=1, keepdims=True)
    return (back * r, bs * r), ((d * n).sum(axis=0), (ds * ns).sum(axis=0)), (d.sum(axis=0), ds.sum(axis=0)), n, ns


def block_norm_grad(dh, dy, h, f, stats, post, gate, scale, col_scale, pre):
    """{"x", "f", "gate", "col_scale", "post_w", "post_b", "pre_w", "pre_b"}: (value, scale) of each."""
    like = dh if dh is not None else dy
    rows, cols = like.shape
    t = np.zeros((rows, cols)) if dh is None else dh
    ts = np.abs(t)
    got = {}
    if dy is not None:
        back, got["pre_w"], got["pre_b"], _, _ = _through(dy, np.abs(dy), h, stats[2:4], pre)
        t, ts = t + back[0], ts + back[1]
    got["x"] = (t, ts)
    if f is None:
        return got
    if post is not None:
        w, b = _ones(post[1], cols), _zeros(post[2], cols)
        n = (f - stats[0][:, None]) * stats[1][:, None]
        z, zs = n * w + b, (np.abs(f) + np.abs(stats[0])[:, None]) * stats[1][:, None] * np.abs(w) + np.abs(b)
    else:
        z, zs = f, np.abs(f)
    a, da = np.ones((1, 1)), None
    if gate is not None:
        access, g, act = _gate(gate, rows)
        a, da = activation(act, g)
    q, qs = t * scale, ts * abs(scale)
    got["col_scale"] = ((q * a * z).sum(axis=0), (qs * np.abs(a) * zs).sum(axis=0))
    c = _ones(col_scale, cols)
    q, qs = q * c, qs * np.abs(c)
    if gate is not None:
        dg, dgs = q * z * da, qs * zs * (np.abs(da) + np.abs(a))
        axis = {"cell": None, "row": 1, "col": 0}[access]
        got["gate"] = (dg, dgs) if axis is None else (dg.sum(axis=axis), dgs.sum(axis=axis))
    d, ds = q * a, qs * np.abs(a)
    if post is not None:
        got["f"], got["post_w"], got["post_b"], _, _ = _through(d, ds, f, stats[0:2], post)
    else:
        got["f"] = (d, ds)
    return got


def grad_norm(grads, kind, max_norm, eps):
    flat = np.concatenate([g.reshape(-1) for g in grads]) if grads else np.zeros(0)
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "l2":
            top = np.abs(flat).max(initial=0.0)
            scaled = flat / top if np.isfinite(top) and top > 0 else flat
            n = np.sqrt((scaled * scaled).sum()) * (top if np.isfinite(top) and top > 0 else 1.0)
        else:
            n = np.abs(flat).max(initial=0.0)
        q = max_norm / (n + eps)
    return n, (1.0 if q >= 1.0 else q)


def adamw(p, g, m, v, factor, lr, betas, eps, step, decay):
    b1, b2 = betas
    g = g * factor
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    p = p - lr * (m / (1.0 - b1 ** step) / (np.sqrt(v / (1.0 - b2 ** step)) + eps) + decay * p)
    return p, m, v
