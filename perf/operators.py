"""The training-step operators as they are measured: what a pass is, on which inputs, and what it cannot do without.

Three operators that a residual block meets in one training step, next to each other:

- block norm: the norm of a block's output, its gate, the residual scale, the addition to the residual stream and the
  norm before the next block, in one pass over the rows ("norm"), and the gradients of all of it ("norm_grad");
- gradient clipping: the global norm of many gradient tensors, the clipping factor, and the clipped gradients ("clip");
- the weight update that takes the clipping factor from the device: AdamW over many tensors, with 32-bit masters and a
  copy of the weights in the block's type ("adamw").

`run` computes a case in plain torch operations in 32 bits, or, with `own` set, through the package's entry points.
"""
import random

import torch

own = False

OPS = ("norm", "norm_grad", "clip", "adamw")
LARGEST = 8192 * 8192          # elements of the largest norm case
BETAS, ADAM_EPS, STEP, LR = (0.9, 0.95), 1e-8, 100, 3e-4
CLIP_EPS = 1e-6


def dt(name):
    return getattr(torch, name)


def size(name):
    return dt(name).itemsize


# ------------------------------------------------------------------------------------------------------------ cases
def norm_case(op, rows, cols, stream, block, post, gate, act, pre, bias=False, residual=True, pad=0, col_scale=False):
    return {"op": op, "rows": rows, "cols": cols, "stream": stream, "block": block, "post": post, "gate": gate,
            "act": act, "pre": pre, "bias": bias, "residual": residual, "pad": pad, "col_scale": col_scale}


def many_case(op, tensors, elements, grad, out, kind="l2"):
    return {"op": op, "tensors": tensors, "elements": elements, "grad": grad, "out": out, "kind": kind}


def listed():
    bf, fl, hf = "bfloat16", "float32", "float16"
    return [
        # one token of a decoding step: post-norm of the block, residual scale, next block's norm; latency alone
        dict(norm_case("norm", 1, 4096, bf, bf, "rms", "none", "linear", "rms", col_scale=True), name="norm one token"),
        # the norm of each attention head's query or key vector: very many short rows, no block and no gate
        dict(norm_case("norm", 131072, 128, bf, bf, "none", "none", "linear", "rms"), name="norm short rows"),
        # an odd model width in padded storage, layer norms with biases, a gate per element
        dict(norm_case("norm", 1531, 1001, hf, hf, "layer", "cell", "silu", "layer", bias=True, pad=23),
             name="norm odd width"),
        # an ordinary training step of a gated block: a token batch of 8192 at width 4096
        dict(norm_case("norm", 8192, 4096, bf, bf, "rms", "cell", "sigmoid", "rms", col_scale=True),
             name="norm training"),
        # a large model: the residual stream in 32 bits, the block in 16
        dict(norm_case("norm", 8192, 8192, fl, bf, "rms", "row", "tanh", "rms"), name="norm wide stream"),
        # a small fine-tuning batch
        dict(norm_case("norm_grad", 64, 2048, bf, bf, "rms", "none", "linear", "rms", col_scale=True),
             name="norm_grad small"),
        # the odd width again, backwards
        dict(norm_case("norm_grad", 1531, 1001, hf, hf, "layer", "cell", "silu", "layer", bias=True, pad=23),
             name="norm_grad odd width"),
        # the training step, backwards: six gradients from one pass
        dict(norm_case("norm_grad", 8192, 4096, bf, bf, "rms", "cell", "sigmoid", "rms", col_scale=True),
             name="norm_grad training"),
        # gradients of low-rank adapters: many small tensors, 32 bits
        dict(many_case("clip", 192, 3_000_000, fl, fl), name="clip adapters"),
        # gradients of whole blocks in 16 bits, clipped into a 32-bit bucket
        dict(many_case("clip", 72, 260_000_000, bf, fl), name="clip blocks"),
        # the adapters' update
        dict(many_case("adamw", 192, 3_000_000, fl, "none"), name="adamw adapters"),
        # the blocks' update: 32-bit masters and moments, 16-bit gradients and weights
        dict(many_case("adamw", 72, 130_000_000, bf, bf), name="adamw blocks"),
    ]


def logint(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choices(OPS, (4, 3, 2, 2))[0]
    if op in ("norm", "norm_grad"):
        stream, block = rng.choice([("bfloat16", "bfloat16"), ("float16", "float16"), ("float32", "float32"),
                                    ("float32", "bfloat16"), ("float32", "float16")])
        cols = logint(rng, 48, 20000)
        if rng.random() < 0.6:                                  # most widths are multiples of 64, some are odd
            cols = max(64, cols // 64 * 64)
        rows = logint(rng, 1, min(131072, LARGEST // 2 // cols))
        post = rng.choice(["none", "rms", "layer"])
        gate = rng.choice(["none", "cell", "row", "col"])
        act = "linear" if gate == "none" else rng.choice(["linear", "sigmoid", "silu", "tanh"])
        plain = post == "none" and gate == "none"
        pre = "rms" if plain else rng.choice(["none", "rms", "layer"])
        return norm_case(op, rows, cols, stream, block, post, gate, act, pre, bias=rng.random() < 0.3,
                         residual=rng.random() < 0.8, pad=rng.choice([0, 0, 0, 8, 64, 3]),
                         col_scale=not plain and rng.random() < 0.4)
    grad = rng.choice(["bfloat16", "float16", "float32"])
    tensors = logint(rng, 1, 400)
    elements = logint(rng, max(20000, 40 * tensors), 130_000_000)
    if op == "clip":
        return many_case(op, tensors, elements, grad, rng.choice([grad, "float32"]), rng.choice(["l2", "l2", "max"]))
    return many_case(op, tensors, elements, grad, "none" if grad == "float32" else grad)


def sizes(case):
    """The tensors' sizes: spread over a factor of about 500 like the matrices, norms and biases of a model, mostly
    multiples of 64, one in eight ragged."""
    rng = random.Random(case["tensors"] * 1_000_003 + case["elements"])
    shares = [500.0 ** rng.random() for _ in range(case["tensors"])]
    total = sum(shares)
    raw = [max(1, int(case["elements"] * s / total)) for s in shares]
    return [n if k % 8 == 5 or n < 64 else n // 64 * 64 for k, n in enumerate(raw)]


def has_block(case):
    """A norm case without a post norm and without a gate is the norm of the stream alone."""
    return case["post"] != "none" or case["gate"] != "none"


# ----------------------------------------------------------------------------------------------------------- inputs
def normal(gen, shape, dtype, spread=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread + mean).to(dt(dtype))


def matrix(gen, case, dtype, spread, channels=None):
    """rows x cols in rows `pad` elements longer; `channels`: a factor per column."""
    full = torch.randn((case["rows"], case["cols"] + case["pad"]), generator=gen, device="cuda").mul_(spread)
    if channels is not None:
        full[:, : case["cols"]] *= channels
    return full.to(dt(dtype))[:, : case["cols"]]


def row_stats(t, kind, eps):
    t = t.float()
    mean = t.mean(1) if kind == "layer" else torch.zeros(t.shape[0], device=t.device)
    var = ((t - mean[:, None]) ** 2).mean(1)
    return mean, 1.0 / torch.sqrt(var + eps)


def prepare_norm(case, gen):
    rows, cols, block = case["rows"], case["cols"], case["block"]
    # a residual stream has a few channels far larger than the rest
    channels = torch.exp(0.7 * torch.randn(cols, generator=gen, device="cuda")).clamp_(max=12.0)
    s = {"case": case, "scale": 0.7, "eps": 1e-6 if case["post"] == "rms" else 1e-5}
    blk = has_block(case)
    s["f"] = matrix(gen, case, block, 0.6) if blk else None
    s["gate"] = None
    if case["gate"] == "cell":
        s["gate"] = matrix(gen, case, block, 1.0)
    elif case["gate"] != "none":
        s["gate"] = normal(gen, (rows if case["gate"] == "row" else cols,), block)
    for part in ("post", "pre"):
        s[part + "_w"] = normal(gen, (cols,), block, 0.1, 1.0) if case[part] != "none" else None
        s[part + "_b"] = normal(gen, (cols,), block, 0.1) if case[part] != "none" and case["bias"] else None
    s["col_scale"] = normal(gen, (cols,), block, 0.2, 0.5) if case["col_scale"] and blk else None
    keeps = not blk or case["residual"]
    if case["op"] == "norm":
        s["x"] = matrix(gen, case, case["stream"], 1.5, channels) if keeps else None
        return s
    s["keeps"] = keeps
    s["h"] = matrix(gen, case, case["stream"], 1.5, channels) if case["pre"] != "none" else None
    s["dy"] = matrix(gen, case, block, 0.02) if case["pre"] != "none" else None
    s["dh"] = matrix(gen, case, case["stream"], 0.02) if keeps or case["pre"] == "none" else None
    # what the forward pass leaves for the backward one: mean and reciprocal spread of the rows of f and of h
    none = (torch.zeros(rows, device="cuda"),) * 2
    fm, fr = row_stats(s["f"], case["post"], s["eps"]) if case["post"] != "none" else none
    hm, hr = row_stats(s["h"], case["pre"], s["eps"]) if case["pre"] != "none" else none
    s["stats"] = torch.stack([fm, fr, hm, hr])
    return s


def packed(ns, flat):
    return list(torch.split(flat, ns))


def prepare_many(case, gen):
    """Gradients are tensors of their own; what is kept over steps lies packed in buckets, tensor behind tensor."""
    ns = sizes(case)
    total = sum(ns)
    s = {"case": case, "g": [normal(gen, (n,), case["grad"], 0.003) for n in ns]}
    if case["op"] == "clip":
        s["out"] = torch.empty(total, dtype=dt(case["out"]), device="cuda")
        s["max_norm"] = 1.0 if case["kind"] == "l2" else 0.005
        s["outs"] = packed(ns, s["out"])
        if own:
            import paper_1801_00829_b200 as fo
            s["list"] = fo.tensor_list(s["g"], s["outs"])
        return s
    s["p"] = normal(gen, (total,), "float32", 0.05)
    s["m"] = normal(gen, (total,), "float32", 0.002)
    s["v"] = normal(gen, (total,), "float32", 0.002).square_()
    s["factor"] = torch.tensor([0.37], device="cuda")
    s["decay"] = [0.1 if n >= 4096 else 0.0 for n in ns]        # norms and biases do not decay
    s["outs"] = [torch.empty(total, device="cuda") for _ in range(3)]
    s["w"] = torch.empty(total, dtype=dt(case["out"]), device="cuda") if case["out"] != "none" else None
    if own:
        import paper_1801_00829_b200 as fo
        p, m, v = (packed(ns, s[k]) for k in ("p", "m", "v"))
        po, mo, vo = (packed(ns, t) for t in s["outs"])
        s["list"] = fo.adam_list(p, s["g"], m, v, decay=s["decay"], outs=(po, mo, vo),
                                 weights=packed(ns, s["w"]) if s["w"] is not None else None)
    else:
        s["decay_flat"] = torch.repeat_interleave(torch.tensor(s["decay"], device="cuda"),
                                                  torch.tensor(ns, device="cuda"), output_size=total)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return prepare_norm(case, gen) if case["op"] in ("norm", "norm_grad") else prepare_many(case, gen)


# ------------------------------------------------------------------------------------------------------ plain forms
def act(kind, g):
    """The gate's activation and its derivative."""
    if kind == "linear":
        return g, torch.ones_like(g)
    if kind == "tanh":
        t = 1.0 - 2.0 / (torch.exp(2.0 * g) + 1.0)
        return t, 1.0 - t * t
    s = 1.0 / (1.0 + torch.exp(-g))
    return (s, s * (1.0 - s)) if kind == "sigmoid" else (g * s, s * (1.0 + g * (1.0 - s)))


def f32(t):
    return None if t is None else t.float()


def gate_of(s):
    """The gate in 32 bits, shaped to broadcast over rows x cols; its activation and derivative."""
    c = s["case"]
    if c["gate"] == "none":
        return None, None
    g = s["gate"].float()
    return act(c["act"], g[:, None] if c["gate"] == "row" else g)


def affine(t, w, b):
    t = t if w is None else t * w.float()
    return t if b is None else t + b.float()


def plain_norm(s):
    c = s["case"]
    h = f32(s["x"])
    if s["f"] is not None:
        z = s["f"].float()
        if c["post"] != "none":
            mean, r = row_stats(z, c["post"], s["eps"])
            z = affine((z - mean[:, None]) * r[:, None], s["post_w"], s["post_b"])
        a, _ = gate_of(s)
        z = z if a is None else z * a
        z = z if s["col_scale"] is None else z * s["col_scale"].float()
        h = z * s["scale"] if h is None else h + z * s["scale"]
    out = [h.to(dt(c["stream"]))] if s["f"] is not None else []
    if c["pre"] != "none":
        mean, r = row_stats(h, c["pre"], s["eps"])
        y = affine((h - mean[:, None]) * r[:, None], s["pre_w"], s["pre_b"])
        out.append(y.to(dt(c["block"])))
    return out


def through_norm(d, t, kind, mean, r, w):
    """The gradient `d` of a norm's output taken through it: to its input, its weight and its bias."""
    n = (t - mean[:, None]) * r[:, None]
    a = d if w is None else d * w.float()
    back = a - n * (a * n).mean(1, keepdim=True)
    if kind == "layer":
        back = back - a.mean(1, keepdim=True)
    return back * r[:, None], (d * n).sum(0), d.sum(0), n


def plain_norm_grad(s):
    c = s["case"]
    fm, fr, hm, hr = s["stats"]
    got = {}
    t = f32(s["dh"])
    if c["pre"] != "none":
        back, dw, db, _ = through_norm(s["dy"].float(), s["h"].float(), c["pre"], hm, hr, s["pre_w"])
        t = back if t is None else t + back
        got["pre_w"] = dw
        if s["pre_b"] is not None:
            got["pre_b"] = db
    if s["keeps"]:
        got["x"] = t.to(dt(c["stream"]))
    if s["f"] is None:
        return got
    f = s["f"].float()
    z = f if c["post"] == "none" else affine((f - fm[:, None]) * fr[:, None], s["post_w"], s["post_b"])
    a, da = gate_of(s)
    q = t * s["scale"]
    if s["col_scale"] is not None:
        got["col_scale"] = (q * (z if a is None else z * a)).sum(0)
        q = q * s["col_scale"].float()
    if a is not None:
        dg = q * z * da
        got["gate"] = dg.to(dt(c["block"])) if c["gate"] == "cell" else dg.sum(1 if c["gate"] == "row" else 0)
        q = q * a
    if c["post"] != "none":
        q, dw, db, _ = through_norm(q, f, c["post"], fm, fr, s["post_w"])
        got["post_w"] = dw
        if s["post_b"] is not None:
            got["post_b"] = db
    got["f"] = q.to(dt(c["block"]))
    return got


def plain_clip(s):
    flat = torch.cat(s["g"]).float()
    norm = torch.sqrt((flat * flat).sum()) if s["case"]["kind"] == "l2" else flat.abs().max()
    factor = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0)
    return [(flat * factor).to(s["out"].dtype), torch.stack([norm, factor])]


def plain_adamw(s):
    b1, b2 = BETAS
    g = torch.cat(s["g"]).float() * s["factor"]
    m = s["m"] * b1 + g * (1.0 - b1)
    v = s["v"] * b2 + g * g * (1.0 - b2)
    step = (m / (1.0 - b1 ** STEP)) / (torch.sqrt(v / (1.0 - b2 ** STEP)) + ADAM_EPS)
    p = s["p"] - LR * (step + s["decay_flat"] * s["p"])
    return [p, m, v] + ([p.to(s["w"].dtype)] if s["w"] is not None else [])


# ------------------------------------------------------------------------------------------------ the package's calls
def own_run(s):
    import paper_1801_00829_b200 as fo
    c = s["case"]
    if c["op"] == "clip":
        result = fo.fused_grad_clip(s["list"], s["max_norm"], kind=c["kind"], eps=CLIP_EPS)
        return [s["out"], result]
    if c["op"] == "adamw":
        fo.fused_adamw(s["list"], lr=LR, betas=BETAS, eps=ADAM_EPS, step=STEP, factor=s["factor"])
        return s["outs"] + ([s["w"]] if s["w"] is not None else [])
    how = {"post": (c["post"], s["post_w"], s["post_b"], s["eps"]) if c["post"] != "none" else None,
           "gate": (c["gate"], s["gate"], c["act"]) if c["gate"] != "none" else None,
           "pre": (c["pre"], s["pre_w"], s["pre_b"], s["eps"]) if c["pre"] != "none" else None,
           "scale": s["scale"], "col_scale": s["col_scale"]}
    if c["op"] == "norm":
        h, y, _ = fo.fused_block_norm(s["x"], s["f"], **how)
        return ([h] if s["f"] is not None else []) + ([y] if y is not None else [])
    return fo.fused_block_norm_grad(s["dh"], s["dy"], s["h"], s["f"], s["stats"], residual=s["keeps"], **how)


def run(state):
    if own:
        return own_run(state)
    return {"norm": plain_norm, "norm_grad": plain_norm_grad, "clip": plain_clip,
            "adamw": plain_adamw}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------------- least work
def work(case):
    if case["op"] in ("clip", "adamw"):
        n = sum(sizes(case))
        if case["op"] == "clip":
            return {"bytes": n * (size(case["grad"]) + size(case["out"])) + 8, "flops": 3 * n}
        low = size(case["out"]) if case["out"] != "none" else 0
        return {"bytes": n * (size(case["grad"]) + 24 + low) + 4, "flops": 16 * n}
    rows, cols = case["rows"], case["cols"]
    cells, ts, tb = rows * cols, size(case["stream"]), size(case["block"])
    blk, pre = has_block(case), case["pre"] != "none"
    keeps = not blk or case["residual"]
    gate = {"none": 0, "cell": cells, "row": rows, "col": cols}[case["gate"]] * tb
    per_norm = cols * tb * (2 if case["bias"] else 1)
    vectors = per_norm * ((case["post"] != "none") + pre) + (cols * tb if case["col_scale"] and blk else 0)
    if case["op"] == "norm":
        moved = cells * ts * (keeps + blk) + cells * tb * (blk + pre) + gate + vectors
        return {"bytes": moved, "flops": cells * (6 * pre + (12 if blk else 0))}
    moved = cells * ts * (2 * keeps + pre + (not keeps and not pre)) + cells * tb * (pre + 2 * blk)
    dgate = cells * tb if case["gate"] == "cell" else gate // tb * 4
    stats = 4 * rows * 2 * ((case["post"] != "none") + pre)
    return {"bytes": moved + gate + dgate + vectors + vectors // tb * 4 + stats,
            "flops": cells * (14 * pre + (24 if blk else 0))}


# ------------------------------------------------------------------------------------------- the definition, 64 bits
def exact_norm(t, kind, eps, w, b):
    if kind == "layer":
        t = t - t.sum(1, keepdim=True) / t.shape[1]
    n = t * torch.rsqrt((t * t).sum(1, keepdim=True) / t.shape[1] + eps)
    n = n * w.double()
    return n if b is None else n + b.double()


def exact_act(kind, g):
    return {"linear": lambda: g, "tanh": lambda: torch.tanh(g), "sigmoid": lambda: torch.sigmoid(g),
            "silu": lambda: g * torch.sigmoid(g)}[kind]()


def exact_forward(s, x, f, gate, vec):
    """(h, y) in 64 bits from 64-bit inputs; `vec`: weights and biases by name."""
    c = s["case"]
    h = x
    if f is not None:
        u = exact_norm(f, c["post"], s["eps"], vec["post_w"], vec["post_b"]) if c["post"] != "none" else f
        if gate is not None:
            u = u * exact_act(c["act"], gate[:, None] if c["gate"] == "row" else gate)
        u = u * s["scale"] * (1.0 if vec["col_scale"] is None else vec["col_scale"])
        h = u if x is None else x + u
    y = exact_norm(h, c["pre"], s["eps"], vec["pre_w"], vec["pre_b"]) if c["pre"] != "none" else None
    return h, y


def wide(t, grad=False):
    return None if t is None else t.double().requires_grad_(grad)


VECTORS = ("post_w", "post_b", "pre_w", "pre_b", "col_scale")


def exact_norm_grad(s):
    """Gradients by reverse differentiation of the definition in 64 bits, at the saved statistics' point: the
    stream's norm is differentiated at h, the block's part at f."""
    c = s["case"]
    vec = {k: wide(s[k], True) for k in VECTORS}
    f, gate, h = wide(s["f"], True), wide(s["gate"], True), wide(s["h"], True)
    t = torch.zeros((c["rows"], c["cols"]), dtype=torch.float64, device="cuda") if s["dh"] is None else s["dh"].double()
    got = {}
    if c["pre"] != "none":
        y = exact_norm(h, c["pre"], s["eps"], vec["pre_w"], vec["pre_b"])
        names = ["pre_w"] + (["pre_b"] if vec["pre_b"] is not None else [])
        g = torch.autograd.grad(y, [h] + [vec[k] for k in names], s["dy"].double())
        t = t + g[0]
        got.update(zip(names, g[1:]))
    if s["keeps"]:
        got["x"] = t
    if f is not None:
        u, _ = exact_forward({**s, "case": {**c, "pre": "none"}}, None, f, gate, vec)
        names = [k for k in ("post_w", "post_b", "col_scale") if vec[k] is not None] + ["f"]
        names += ["gate"] if gate is not None else []
        leaves = [{"f": f, "gate": gate, **vec}[k] for k in names]
        got.update(zip(names, torch.autograd.grad(u, leaves, t)))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        vec = {k: wide(s[k]) for k in VECTORS}
        h, y = exact_forward(s, wide(s["x"]), wide(s["f"]), wide(s["gate"]), vec)
        return ([h] if s["f"] is not None else []) + ([y] if y is not None else [])
    if case["op"] == "norm_grad":
        return exact_norm_grad(s)
    g = torch.cat([t.double() for t in s["g"]])
    if case["op"] == "clip":
        norm = torch.linalg.vector_norm(g) if case["kind"] == "l2" else torch.amax(torch.abs(g))
        factor = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0)
        return [g * factor, torch.stack([norm, factor])]
    b1, b2 = BETAS
    g = g * s["factor"].double()
    m = b1 * s["m"].double() + (1.0 - b1) * g
    v = b2 * s["v"].double() + (1.0 - b2) * g ** 2
    p = s["p"].double()
    decay = torch.cat([torch.full((t.numel(),), d, dtype=torch.float64, device="cuda")
                       for t, d in zip(s["g"], s["decay"])])
    p = p * (1.0 - LR * decay) - LR * (m / (1.0 - b1 ** STEP)) / ((v / (1.0 - b2 ** STEP)) ** 0.5 + ADAM_EPS)
    return [p, m, v] + ([p.clone()] if s["w"] is not None else [])
