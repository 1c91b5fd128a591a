"""More operators of a language model's step as they are measured: what a pass is, on which inputs, and what it cannot do
without.

Three that a model meets beside its block norms, each forward and backward:

- head norms with the position rotation: the norm of every head's query and key vector and the rotation by its token's
  position, which may have several axes (time, height, width), in one pass over both tensors ("heads");
- a gated linear recurrence over the tokens, h_t = a_t h_{t-1} + m(a_t) x_t, with states, padded batches and document
  borders, down to a single token ("scan");
- the distillation loss from a teacher's top logits over a vocabulary, its gradient, and both in one pass ("distill").

`run` computes a case in plain torch operations in 32 bits, or, with `own` set, through the package's entry points.
"""
import math

import torch

own = False

LARGEST = 4096 * 128000          # logits of the largest distillation case
SCAN_LARGEST = 65536 * 2560      # elements of the largest recurrence case
HEADS_LARGEST = 8192 * 40 * 128  # elements of the largest case of head norms
EPS = 1e-6


def dt(name):
    return getattr(torch, name)


def size(name):
    return dt(name).itemsize


# ------------------------------------------------------------------------------------------------------------ cases
def heads_case(way, batch, tokens, hq, hk, d, rot, pairing, kind, dtype="bfloat16", sections="", bias=False, layout="packed"):
    return {"op": "heads", "way": way, "batch": batch, "tokens": tokens, "hq": hq, "hk": hk, "d": d, "rot": rot,
            "pairing": pairing, "kind": kind, "type": dtype, "sections": sections, "bias": bias, "layout": layout}


def scan_case(way, batch, tokens, channels, dtype, gate, decay, mix, state=False, reset=False, lengths=False, pad=0):
    return {"op": "scan", "way": way, "batch": batch, "tokens": tokens, "channels": channels, "type": dtype, "gate": gate,
            "decay": decay, "mix": mix, "state": state, "reset": reset, "lengths": lengths, "pad": pad}


def distill_case(way, rows, vocab, top, dtype, tail, temperature, ids="int64", values="float32", pad=0):
    return {"op": "distill", "way": way, "rows": rows, "vocab": vocab, "top": top, "type": dtype, "tail": tail,
            "temperature": temperature, "ids": ids, "values": values, "pad": pad}


def listed():
    bf, fl, hf = "bfloat16", "float32", "float16"
    return [
        # one new token of 4 sequences in a decoding step: latency alone
        dict(heads_case("forward", 4, 1, 32, 8, 128, 128, "halves", "rms"), name="heads one token"),
        # a training batch of text with shared key heads, views into the packed projection
        dict(heads_case("forward", 4, 2048, 32, 8, 128, 128, "halves", "rms"), name="heads training"),
        # video tokens with three axes, an odd head size in 16-bit floats, neighbouring pairs, from attention in heads-first
        # order, backwards
        dict(heads_case("backward", 1, 7605, 12, 12, 72, 72, "pairs", "layer", hf, "12,12,12", True, "heads_first"),
             name="heads video backward"),
        # the training batch, backwards
        dict(heads_case("backward", 4, 2048, 32, 8, 128, 128, "halves", "rms"), name="heads training backward"),
        # one new token of 64 sequences with their states
        dict(scan_case("forward", 64, 1, 4096, bf, bf, "sigmoid", "rest", state=True), name="scan one token"),
        # a training batch
        dict(scan_case("forward", 8, 4096, 2048, bf, bf, "sigmoid", "rest"), name="scan training"),
        # one long document with decays in 32 bits, as logarithms
        dict(scan_case("forward", 1, 65536, 2560, bf, fl, "exp", "root"), name="scan long"),
        # a ragged batch of padded sequences with document borders in them, an odd width, backwards
        dict(scan_case("backward", 5, 777, 1001, fl, fl, "sigmoid", "root", True, True, True, 7), name="scan ragged backward"),
        # the training batch, backwards
        dict(scan_case("backward", 8, 4096, 2048, bf, bf, "sigmoid", "rest"), name="scan training backward"),
        # an evaluation of a few rows over an odd vocabulary in 32 bits, the teacher's entries alone
        dict(distill_case("loss", 37, 50257, 10, fl, False, 1.0), name="distill evaluation"),
        # the gradient alone, where the loss was computed in the forward pass
        dict(distill_case("gradient", 2048, 32000, 32, hf, True, 1.0, "int32", hf), name="distill backward"),
        # a training batch over a large vocabulary: loss and gradient, with the teacher's remaining mass
        dict(distill_case("step", 4096, 128000, 64, bf, True, 2.0), name="distill training"),
    ]


def logint(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw_heads(rng):
    way = rng.choice(["forward", "backward"])
    d = rng.choice([64, 128, 128, 256, rng.choice([72, 80, 96, 192]), rng.randrange(16, 257)])
    rot = rng.choice([d, d, d, d // 2, d // 4]) // 2 * 2
    hq = rng.choice([1, 4, 8, 12, 16, 32, 40, rng.randrange(1, 65)])
    hk = rng.choice([0, 1, hq, hq, max(1, hq // 4)])
    batch = rng.choice([1, 1, 2, 4, 16])
    tokens = logint(rng, 1, max(1, HEADS_LARGEST // (batch * (hq + hk) * d)))
    kind = rng.choice(["rms", "rms", "layer", "none"])
    sections = ""
    if rng.random() < 0.35 and rot >= 8:
        first, second = rot // 8, (rot // 2 - rot // 8) // 2
        sections = "%d,%d,%d" % (first, second, rot // 2 - first - second)
    return heads_case(way, batch, tokens, hq, hk, d, rot, rng.choice(["halves", "halves", "pairs"]), kind,
                      rng.choice(["bfloat16", "bfloat16", "float16", "float32"]), sections,
                      kind != "none" and rng.random() < 0.3, rng.choice(["packed", "packed", "plain", "heads_first"]))


def draw_scan(rng):
    way = rng.choice(["forward", "forward", "backward"])
    dtype, gate = rng.choice([("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float16"),
                              ("float16", "float32"), ("float32", "float32")])
    channels = logint(rng, 16, 8192)
    if rng.random() < 0.7:
        channels = max(32, channels // 32 * 32)
    batch = logint(rng, 1, 64)
    most = SCAN_LARGEST // 2 // (batch * channels)
    tokens = rng.choice([1, logint(rng, 2, max(2, min(65536, most))), logint(rng, 2, max(2, min(65536, most)))])
    decay = rng.choice(["sigmoid", "exp", "value"])
    return scan_case(way, batch, tokens, channels, dtype, gate, decay, rng.choice(["one", "rest", "root"]),
                     rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.3, rng.choice([0, 0, 0, 64, 3]))


def draw_distill(rng):
    way = rng.choice(["loss", "gradient", "step"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    vocab = rng.choice([32000, 50257, 65536, 100003, 128000, logint(rng, 300, 200000)])
    rows = logint(rng, 1, max(1, min(16384, LARGEST // 2 // vocab)))
    return distill_case(way, rows, vocab, rng.choice([1, 8, 20, 64, 128, min(vocab, 256)]), dtype, rng.random() < 0.6,
                        rng.choice([1.0, 1.0, 2.0, 0.7]), rng.choice(["int64", "int32"]), rng.choice(["float32", dtype]),
                        rng.choice([0, 0, 0, 64, 5]))


def draw(rng):
    return rng.choice([draw_heads, draw_scan, draw_distill])(rng)


# ----------------------------------------------------------------------------------------------------------- inputs
def normal(gen, shape, dtype, spread=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread + mean).to(dt(dtype))


def uniform(gen, shape):
    return torch.rand(shape, generator=gen, device="cuda")


def sections_of(case):
    return tuple(int(n) for n in case["sections"].split(",")) if case["sections"] else None


def head_tensors(gen, case, spread):
    """Queries and keys (batch, tokens, heads, d) as the program has them: views into one packed projection, tensors of
    their own, or the order that attention works in (heads before tokens)."""
    b, t, hq, hk, d = (case[k] for k in ("batch", "tokens", "hq", "hk", "d"))
    # a few channels of queries and keys are far larger than the rest
    channels = torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda")).clamp_(max=8.0)

    def one(shape):
        return (torch.randn(shape, generator=gen, device="cuda") * spread * channels).to(dt(case["type"]))
    if case["layout"] == "packed":
        both = one((b, t, hq + 2 * hk, d))                      # queries, keys, values
        return both[:, :, :hq], both[:, :, hq:hq + hk] if hk else None
    if case["layout"] == "heads_first":
        return tuple(one((b, h, t, d)).transpose(1, 2) if h else None for h in (hq, hk))
    return tuple(one((b, t, h, d)) if h else None for h in (hq, hk))


def prepare_heads(case, gen):
    s = {"case": case}
    b, t, d, pairs = case["batch"], case["tokens"], case["d"], case["rot"] // 2
    s["q"], s["k"] = head_tensors(gen, case, 1.3)
    for part in ("q", "k"):
        given = case["kind"] != "none" and s[part] is not None
        s[part + "_w"] = normal(gen, (d,), case["type"], 0.15, 1.0) if given else None
        s[part + "_b"] = normal(gen, (d,), case["type"], 0.1) if given and case["bias"] else None
    sections = sections_of(case)
    if sections:
        # a grid of frames: time, height and width of each token
        side = max(1, int(math.sqrt(t / 5)))
        at = torch.arange(t, device="cuda")
        grid = torch.stack([at // (side * side), at // side % side, at % side])
        s["positions"] = grid[:, None, :].expand(3, b, t)
        longest = max(side, (t - 1) // (side * side) + 1)
    else:
        # each sequence of the batch is somewhere else in its text
        start = torch.randint(0, 4096, (b, 1), generator=gen, device="cuda")
        s["positions"] = start + torch.arange(t, device="cuda")
        longest = 4096 + t
    if pairs:
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None]
        angle = angle * 10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
        s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    if case["way"] == "backward":
        s["dq"], s["dk"] = head_tensors(gen, {**case, "layout": "heads_first" if case["layout"] == "heads_first" else "plain"}, 0.02)
    return s


def prepare_scan(case, gen):
    b, t, c, pad = (case[k] for k in ("batch", "tokens", "channels", "pad"))
    s = {"case": case}

    def one(dtype, spread, mean=0.0):
        return normal(gen, (b, t, c + pad), dtype, spread, mean)[:, :, :c]
    s["x"] = one(case["type"], 1.0)
    # decays near one, spread over the channels as trained gates are
    slow = torch.randn(c, generator=gen, device="cuda")
    g = torch.randn((b, t, c + pad), generator=gen, device="cuda")
    g[:, :, :c] += 2.5 + 1.5 * slow
    if case["decay"] == "value":
        g = (1.0 / (1.0 + torch.exp(-g))).clamp_(max=0.98)      # a decay of 1 has no slope under the root
    elif case["decay"] == "exp":
        g = -0.3 * torch.log1p(torch.exp(-g))
    s["gate"] = g.to(dt(case["gate"]))[:, :, :c]
    del g
    s["state"] = torch.randn((b, c), generator=gen, device="cuda") if case["state"] else None
    s["reset"] = uniform(gen, (b, t)) < 0.005 if case["reset"] else None
    s["lengths"] = None
    if case["lengths"]:
        s["lengths"] = (uniform(gen, (b,)) * (t + 1)).long().clamp_(max=t)
        s["lengths"][0] = t
    if case["way"] == "backward":
        s["h"] = plain_scan(s)[0]
        s["dh"] = one(case["type"], 0.02)
        s["dlast"] = normal(gen, (b, c), "float32", 0.02) if case["state"] else None
    return s


def prepare_distill(case, gen):
    rows, vocab, top, pad = (case[k] for k in ("rows", "vocab", "top", "pad"))
    s = {"case": case}
    s["logits"] = normal(gen, (rows, vocab + pad), case["type"], 2.5)[:, :vocab]
    # the teacher is surer than the student, and mostly agrees with it
    teacher = torch.randn((rows, vocab), generator=gen, device="cuda").add_(s["logits"].float(), alpha=1.1)
    values, ids = teacher.topk(top, dim=1)
    s["ids"], s["values"] = ids.to(dt(case["ids"])), values.to(dt(case["values"]))
    s["tail"] = None
    if case["tail"]:
        teacher.scatter_(1, ids, s["values"].float())
        s["tail"] = torch.logsumexp(teacher.div_(case["temperature"]), 1)
    del teacher
    # the mean over the tokens that count: prompts and padding, one in six, do not
    counts = uniform(gen, (rows,)) > 1 / 6
    s["dloss"] = counts / counts.sum().clamp(min=1)
    if case["type"] == "float16":
        s["dloss"] *= 32768.0                                   # the loss scale that gradients of this type need
    if case["way"] == "gradient":
        most, total, ratio = student(s)[:3]
        s["stats"] = torch.stack([most.double(), total, 1.0 - ratio]).float()    # as the forward pass leaves them
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"heads": prepare_heads, "scan": prepare_scan, "distill": prepare_distill}[case["op"]](case, gen)


# ------------------------------------------------------------------------------------------------------ plain forms
def f32(t):
    return None if t is None else t.float()


def angles(s):
    """Cosines and sines of every token's pairs, shaped to broadcast over the heads."""
    sections = sections_of(s["case"])
    if not sections:
        return s["cos"][s["positions"]][:, :, None], s["sin"][s["positions"]][:, :, None]
    axis = torch.repeat_interleave(torch.arange(len(sections), device="cuda"), torch.tensor(sections, device="cuda"))
    at, pair = s["positions"][axis].permute(1, 2, 0), torch.arange(len(axis), device="cuda")
    return s["cos"][at, pair][:, :, None], s["sin"][at, pair][:, :, None]


def turned(t, case, cos, sin):
    rot, out = case["rot"], t.clone()
    if case["pairing"] == "halves":
        a, b = t[..., :rot // 2], t[..., rot // 2:rot]
        out[..., :rot // 2], out[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = t[..., 0:rot:2], t[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return out


def normed(t, kind):
    """(t - mean) * r and r of every head's vector."""
    if kind == "none":
        return t, None
    if kind == "layer":
        t = t - t.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS)
    return t * r, r


def plain_heads(s):
    c = s["case"]
    cos, sin = angles(s) if c["rot"] else (None, None)
    out = {}
    for part in ("q", "k"):
        if s[part] is None:
            continue
        n, r = normed(s[part].float(), c["kind"])
        w, b = f32(s[part + "_w"]), f32(s[part + "_b"])
        if c["way"] == "forward":
            y = n if w is None else n * w
            y = y if b is None else y + b
            out[part] = (turned(y, c, cos, sin) if c["rot"] else y).to(s[part].dtype)
            continue
        g = s["d" + part].float()
        g = turned(g, c, cos, -sin) if c["rot"] else g
        if w is not None:
            out[part + "_w"] = (g * n).sum((0, 1, 2))
        if b is not None:
            out[part + "_b"] = g.sum((0, 1, 2))
        if r is not None:
            a = g * w
            g = a - n * (a * n).mean(-1, keepdim=True)
            if c["kind"] == "layer":
                g = g - a.mean(-1, keepdim=True)
            g = g * r
        out[part] = g.to(s[part].dtype)
    return out


def decays(s):
    """a and 1 - a in 32 bits, the latter without the cancellation."""
    g = s["gate"].float()
    if s["case"]["decay"] == "value":
        return g, 1.0 - g
    if s["case"]["decay"] == "exp":
        return torch.exp(g), -torch.expm1(g)
    return 1.0 / (1.0 + torch.exp(-g)), 1.0 / (1.0 + torch.exp(g))


def mixed(s, a, rest):
    mix = s["case"]["mix"]
    return torch.ones_like(a) if mix == "one" else rest if mix == "rest" else torch.sqrt(rest * (1.0 + a))


def behind(s):
    """True at places behind a sequence's end, (batch, tokens, 1); None without lengths."""
    if s["lengths"] is None:
        return None
    return (torch.arange(s["case"]["tokens"], device="cuda") >= s["lengths"][:, None])[:, :, None]


def carries(s, a):
    """What the state is multiplied by from token to token: nothing crosses a border, and behind the end it stays."""
    if s["reset"] is not None:
        a = a.masked_fill(s["reset"][:, :, None], 0.0)
    return a if s["lengths"] is None else a.masked_fill(behind(s), 1.0)


def recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from h = 0, in as many steps as the length has bits."""
    step = 1
    while step < a.shape[1]:
        b = torch.cat([b[:, :step], torch.addcmul(b[:, step:], a[:, step:], b[:, :-step])], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def plain_scan(s):
    a, rest = decays(s)
    b = mixed(s, a, rest) * s["x"].float()
    end = behind(s)
    a = carries(s, a)
    if end is not None:
        b = b.masked_fill(end, 0.0)
    if s["state"] is not None:
        b[:, 0] += a[:, 0] * s["state"]
    h = recurrence(a, b)
    last = h[:, -1].clone()
    return [(h if end is None else h.masked_fill(end, 0.0)).to(s["x"].dtype), last]


def plain_scan_grad(s):
    c = s["case"]
    a, rest = decays(s)
    x, mix, end, keep = s["x"].float(), mixed(s, a, rest), behind(s), carries(s, a)
    d = s["dh"].float()
    if end is not None:
        d = d.masked_fill(end, 0.0)
    if s["dlast"] is not None:
        d = torch.cat([d[:, :-1], d[:, -1:] + s["dlast"][:, None]], 1)
    # the recurrence backwards: what reaches token t comes through the decay of token t + 1
    after = torch.cat([keep[:, 1:], torch.zeros_like(keep[:, :1])], 1)
    lam = recurrence(after.flip(1), d.flip(1)).flip(1)
    first = torch.zeros_like(x[:, 0]) if s["state"] is None else s["state"]
    before = torch.cat([first[:, None], s["h"].float()[:, :-1]], 1)
    if s["reset"] is not None:
        before = before.masked_fill(s["reset"][:, :, None], 0.0)
    slope = {"value": torch.ones_like(a), "exp": a, "sigmoid": a * rest}[c["decay"]]
    dmix = {"one": torch.zeros_like(a), "rest": -slope, "root": -a * slope / mix}[c["mix"]]
    dx, dg = lam * mix, lam * (slope * before + dmix * x)
    if end is not None:
        dx, dg = dx.masked_fill(end, 0.0), dg.masked_fill(end, 0.0)
    got = {"x": dx.to(s["x"].dtype), "gate": dg.to(s["gate"].dtype)}
    if s["state"] is not None:
        got["state"] = keep[:, 0] * lam[:, 0]
    return got


def shares(s):
    """The teacher's shares of its entries, and of all the rest (None: the entries are all there is)."""
    t = s["values"].double() / s["case"]["temperature"]
    if s["tail"] is None:
        e = torch.exp(t - t.amax(1, keepdim=True))
        return e / e.sum(1, keepdim=True), None
    p = torch.exp(t - s["tail"].double()[:, None])
    return p, (1.0 - p.sum(1)).clamp(min=0.0)


def student(s):
    """Of every row: the largest logit, the sum of exp((z - largest) / temperature), and the teacher's rest over the
    student's; the entries' scaled distances from the largest, the teacher's shares.  The entries are taken in 64 bits: they
    hold most of the sum, and the loss is a difference of logarithms."""
    inverse, ids = 1.0 / s["case"]["temperature"], s["ids"].long()
    z = s["logits"].float()
    most = z.amax(1)
    at = (z.gather(1, ids).double() - most[:, None]) * inverse
    p, rest = shares(s)
    others = torch.exp((z - most[:, None]).mul_(inverse)).scatter_(1, ids, 0.0).sum(1).double()
    total = others + torch.exp(at).sum(1)
    ratio = torch.zeros_like(total) if rest is None else rest * total / others
    return most, total, ratio, at, p, rest


def plain_loss(s, total, ratio, at, p, rest):
    each = p * (torch.log(p) - at + torch.log(total)[:, None])
    loss = torch.where(p > 0, each, torch.zeros_like(each)).sum(1)
    if rest is not None:
        loss = loss + torch.where(rest > 0, rest * torch.log(ratio), torch.zeros_like(rest))
    return loss.float()


def plain_gradient(s, most, total, factor, p):
    """factor: what a probability outside the teacher's entries is multiplied by."""
    ids, inverse = s["ids"].long(), 1.0 / s["case"]["temperature"]
    q = torch.exp((s["logits"].float() - most[:, None]).mul_(inverse)) / total[:, None]
    inside = q.gather(1, ids) - p.float()
    d = (q * factor[:, None]).scatter_(1, ids, inside) * (s["dloss"] * inverse)[:, None]
    return d.to(s["logits"].dtype)


def plain_distill(s):
    way = s["case"]["way"]
    if way == "gradient":
        most, total, factor = s["stats"]
        return [plain_gradient(s, most, total, factor, shares(s)[0])]
    most, total, ratio, at, p, rest = student(s)
    loss = plain_loss(s, total, ratio, at, p, rest)
    if way == "loss":
        return [loss]
    # a row that does not count has no loss either
    return [torch.where(s["dloss"] != 0, loss, torch.zeros_like(loss)),
            plain_gradient(s, most, total.float(), (1.0 - ratio).float(), p)]


# ------------------------------------------------------------------------------------------------ the package's calls
def own_heads(s):
    import paper_1801_00829_b200 as fo
    c = s["case"]
    how = {part + "_norm": (c["kind"], s[part + "_w"], s[part + "_b"], EPS) if s[part + "_w"] is not None else None
           for part in ("q", "k")}
    how["rotate"] = (s["cos"], s["sin"], s["positions"], c["pairing"], sections_of(c)) if c["rot"] else None
    if c["way"] == "backward":
        return fo.fused_head_norm_grad(s["dq"], s["dk"], s["q"], s["k"], **how)
    q, k = fo.fused_head_norm(s["q"], s["k"], **how)
    return {"q": q} if k is None else {"q": q, "k": k}


def own_scan(s):
    import paper_1801_00829_b200 as fo
    c = s["case"]
    how = {"decay": c["decay"], "mix": c["mix"], "state": s["state"], "reset": s["reset"], "lengths": s["lengths"]}
    if c["way"] == "backward":
        return fo.fused_scan_grad(s["dh"], s["x"], s["gate"], s["h"], dlast=s["dlast"], **how)
    return fo.fused_scan(s["x"], s["gate"], **how)


def own_distill(s):
    import paper_1801_00829_b200 as fo
    way, how = s["case"]["way"], {"tail": s["tail"], "temperature": s["case"]["temperature"]}
    if way == "loss":
        return [fo.fused_distill(s["logits"], s["ids"], s["values"], **how)[0]]
    if way == "gradient":
        return [fo.fused_distill_grad(s["dloss"], s["logits"], s["ids"], s["values"], s["stats"], **how)]
    return fo.fused_distill_step(s["dloss"], s["logits"], s["ids"], s["values"], **how)


def run(state):
    c = state["case"]
    if own:
        return {"heads": own_heads, "scan": own_scan, "distill": own_distill}[c["op"]](state)
    if c["op"] == "scan":
        return plain_scan_grad(state) if c["way"] == "backward" else plain_scan(state)
    return plain_heads(state) if c["op"] == "heads" else plain_distill(state)


# ------------------------------------------------------------------------------------------------------- least work
def work(case):
    if case["op"] == "heads":
        tokens, heads = case["batch"] * case["tokens"], case["hq"] + case["hk"]
        cells, axes = tokens * heads * case["d"], 3 if case["sections"] else 1
        vectors = 0 if case["kind"] == "none" else case["d"] * (2 if case["hk"] else 1) * (2 if case["bias"] else 1)
        places = tokens * (8 * axes + 4 * case["rot"]) if case["rot"] else 0      # positions, cosines and sines
        if case["way"] == "forward":
            return {"bytes": 2 * cells * size(case["type"]) + vectors * size(case["type"]) + places, "flops": 9 * cells}
        moved = 2 if case["kind"] == "none" else 3                                # without a norm q and k are not needed
        return {"bytes": moved * cells * size(case["type"]) + vectors * (size(case["type"]) + 4) + places, "flops": 19 * cells}
    if case["op"] == "scan":
        rows = case["batch"] * case["tokens"]
        cells, st = rows * case["channels"], 4 * case["batch"] * case["channels"]
        marks = rows * case["reset"] + 8 * case["batch"] * case["lengths"]
        te, tg = size(case["type"]), size(case["gate"])
        if case["way"] == "forward":
            return {"bytes": cells * (2 * te + tg) + st * (1 + case["state"]) + marks, "flops": 8 * cells}
        read = 2 if case["mix"] == "one" else 3                                       # x only where the decay mixes it in
        return {"bytes": cells * ((read + 1) * te + 2 * tg) + 3 * st * case["state"] + marks, "flops": 16 * cells}
    cells, entries = case["rows"] * case["vocab"], case["rows"] * case["top"]
    moved = cells * size(case["type"]) * (1 if case["way"] == "loss" else 2)
    moved += entries * (size(case["ids"]) + size(case["values"]))
    per_row = 4 * (case["tail"] + (case["way"] != "loss") + (3 if case["way"] == "gradient" else 1))
    return {"bytes": moved + case["rows"] * per_row, "flops": cells * {"loss": 4, "gradient": 4, "step": 8}[case["way"]]}


# ------------------------------------------------------------------------------------------- the definition, 64 bits
def wide(t, grad=False):
    return None if t is None else t.double().requires_grad_(grad)


def exact_head(s, part, t, w, b):
    """The definition with complex numbers: a pair is turned by its token's angle."""
    c = s["case"]
    if c["kind"] == "layer":
        t = torch.nn.functional.layer_norm(t, (c["d"],), w, b, EPS)
    elif c["kind"] == "rms":
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w
        t = t if b is None else t + b
    if not c["rot"]:
        return t
    pairs, at, first = c["rot"] // 2, [], 0
    sections = sections_of(c) or (pairs,)
    places = s["positions"] if c["sections"] else s["positions"][None]
    for n, place in zip(sections, places):
        unit = torch.complex(s["cos"].double(), s["sin"].double())[:, first:first + n]
        at.append(unit[place])
        first += n
    unit = torch.cat(at, -1)[:, :, None]
    body, plain = t[..., :c["rot"]], t[..., c["rot"]:]
    if c["pairing"] == "pairs":
        body = torch.view_as_real(torch.view_as_complex(body.unflatten(-1, (pairs, 2)).contiguous()) * unit).flatten(-2)
    else:
        z = torch.complex(*body.unflatten(-1, (2, pairs)).unbind(-2)) * unit
        body = torch.cat([z.real, z.imag], -1)
    return torch.cat([body, plain], -1)


def exact_heads(s):
    out = {}
    for part in ("q", "k"):
        if s[part] is None:
            continue
        back = s["case"]["way"] == "backward"
        leaves = {name: wide(s[name], back) for name in (part, part + "_w", part + "_b") if s[name] is not None}
        y = exact_head(s, part, leaves[part], leaves.get(part + "_w"), leaves.get(part + "_b"))
        if back:
            out.update(zip(leaves, torch.autograd.grad(y, list(leaves.values()), s["d" + part].double())))
        else:
            out[part] = y
    return out


def exact_decay(s):
    g = s["gate"].double()
    kind = s["case"]["decay"]
    log = torch.log(g) if kind == "value" else g if kind == "exp" else torch.nn.functional.logsigmoid(g)
    a, rest = torch.exp(log), -torch.expm1(log)
    if kind == "value":
        a, rest = g, 1.0 - g
    mix = s["case"]["mix"]
    m = torch.ones_like(a) if mix == "one" else rest if mix == "rest" else torch.sqrt(rest * (2.0 - rest))
    return a, rest, m


def exact_scan(s):
    """Token after token."""
    a, _, m = exact_decay(s)
    b = m * s["x"].double()
    batch, tokens, channels = a.shape
    length = torch.full((batch,), tokens, device="cuda") if s["lengths"] is None else s["lengths"]
    drops = torch.zeros((batch, tokens), dtype=torch.bool, device="cuda") if s["reset"] is None else s["reset"]
    simple = s["lengths"] is None and s["reset"] is None
    h = torch.zeros((batch, channels), dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    out = torch.zeros_like(a)
    for t in range(tokens):
        if simple:
            h = torch.addcmul(b[:, t], a[:, t], h)
            out[:, t] = h
            continue
        new = torch.where(drops[:, t, None], b[:, t], a[:, t] * h + b[:, t])
        on = (t < length)[:, None]
        h = torch.where(on, new, h)
        out[:, t] = torch.where(on, new, torch.zeros_like(new))
    return [out, h]


def exact_scan_grad(s):
    """Backwards token after token, from the chain rule at the saved states."""
    c = s["case"]
    a, rest, m = exact_decay(s)
    batch, tokens, channels = a.shape
    x, h, d = s["x"].double(), s["h"].double(), s["dh"].double()
    start = torch.zeros((batch, channels), dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    length = torch.full((batch,), tokens, device="cuda") if s["lengths"] is None else s["lengths"]
    da = {"value": torch.ones_like(a), "exp": a, "sigmoid": a * rest}[c["decay"]]
    dm = {"one": torch.zeros_like(a), "rest": -da, "root": -da * a / m}[c["mix"]]
    carry = torch.zeros_like(start) if s["dlast"] is None else s["dlast"].double()
    dx, dg = torch.zeros_like(a), torch.zeros_like(a)
    none = torch.zeros_like(start)
    for t in reversed(range(tokens)):
        on = (t < length)[:, None]
        lam = carry + d[:, t]
        before = h[:, t - 1] if t else start
        through = a[:, t] * lam
        if s["reset"] is not None:
            drop = s["reset"][:, t, None]
            before, through = torch.where(drop, none, before), torch.where(drop, none, through)
        dx[:, t] = torch.where(on, m[:, t] * lam, none)
        dg[:, t] = torch.where(on, lam * (da[:, t] * before + dm[:, t] * x[:, t]), none)
        carry = torch.where(on, through, carry)
    got = {"x": dx, "gate": dg}
    if s["state"] is not None:
        got["state"] = carry
    return got


def exact_distill(s):
    """The divergence of the teacher's shares from the student's: over the entries and, with the teacher's total, one
    more share for everything else."""
    c = s["case"]
    ids, t = s["ids"].long(), s["values"].double() / c["temperature"]
    p = torch.softmax(t, 1) if s["tail"] is None else torch.exp(t - s["tail"].double()[:, None])
    z = s["logits"].double() / c["temperature"]
    logq = torch.log_softmax(z, 1)
    inside = torch.zeros_like(z, dtype=torch.bool).scatter_(1, ids, True)
    loss = (torch.special.xlogy(p, p) - p * logq.gather(1, ids)).sum(1)
    share = torch.ones_like(loss)
    if s["tail"] is not None:
        rest = (1.0 - p.sum(1)).clamp(min=0.0)
        logrest = torch.logsumexp(logq.masked_fill(inside, -math.inf), 1)
        loss = loss + torch.special.xlogy(rest, rest) - torch.where(rest > 0, rest * logrest, torch.zeros_like(rest))
        share = 1.0 - rest / torch.exp(logrest)
    if c["way"] == "loss":
        return [loss]
    counts = s["dloss"] != 0
    d = logq.exp_()
    d = torch.where(inside, d, d * share[:, None])
    d.scatter_add_(1, ids, -p)
    d *= (s["dloss"].double() / c["temperature"])[:, None]
    return [d] if c["way"] == "gradient" else [torch.where(counts, loss, torch.zeros_like(loss)), d]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "scan":
        return exact_scan_grad(s) if case["way"] == "backward" else exact_scan(s)
    return exact_heads(s) if case["op"] == "heads" else exact_distill(s)
