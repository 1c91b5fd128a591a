"""Head norms with rotation, the gated recurrence and the distillation loss against plain float64 evaluations (oracle/lm.py), at
the sizes, types, layouts, masks and values where they can go wrong.

Tolerances.  A result is rounded once to its type (relative u, plus half the smallest subnormal); before that every operation rounds
to 32 bits (64 for float64).
- heads: a value passes a sum over its head, a reciprocal root and about a dozen products: 64 units of the magnitude it was
  added up from; sums over n vectors n units more.
- recurrence: the oracle carries a bound along, token by token (the error of the decay, of m(a), and of each rounding).
- distillation: the rest's sum is off by at most a unit per addition of a thread and 12 + 2 |exponent| units per term (the weight
  exp(-|exponent|) keeps the second below 16); q, the loss and the factor follow from that.
"""
import numpy as np
import pytest
import torch

import paper_1801_00829_b200 as fo
from oracle import lm as ref

pytestmark = pytest.mark.gpu

F64, F32, BF16, F16 = torch.float64, torch.float32, torch.bfloat16, torch.float16
TYPES = [F64, F32, BF16, F16]
ROUND = {F64: (2.0 ** -53, 0.0), F32: (2.0 ** -24, 2.0 ** -126), BF16: (2.0 ** -8, 2.0 ** -126), F16: (2.0 ** -11, 2.0 ** -25)}


def unit(t):
    return 2.0 ** -53 if t == F64 else 2.0 ** -24


def wide(t):
    return F64 if t == F64 else F32


def host(t):
    return None if t is None else t.detach().to(F64 if t.is_floating_point() else t.dtype).cpu().numpy()


def close(got, want, error, what):
    """error: before the rounding to got's type."""
    rel, least = ROUND[got.dtype]
    g = host(got)
    assert g.shape == want.shape, "%s: shape %s, not %s" % (what, g.shape, want.shape)
    with np.errstate(invalid="ignore"):
        limit = rel * np.abs(want) + least + error * (1.0 + rel)
        ok = (np.abs(g - want) <= limit) | (np.isnan(want) & np.isnan(g)) | (np.isinf(want) & (g == want))
    assert ok.all(), "%s: %d of %d off, first %r for %r (limit %r)" % (
        what, (~ok).sum(), ok.size, g[~ok].flat[0], want[~ok].flat[0], np.broadcast_to(limit, ok.shape)[~ok].flat[0])


def made(rng, shape, dtype, spread=1.0, mean=0.0, pad=0, shift=0):
    """A tensor whose rows are `pad` elements longer than they look and begin `shift` elements into the storage."""
    full = rng.randn(*shape[:-1], shape[-1] + pad) * spread + mean
    flat = torch.zeros(full.size + shift, dtype=dtype, device="cuda")
    flat[shift:] = torch.from_numpy(full.reshape(-1)).to(dtype).cuda()
    return flat[shift:].view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]


# ------------------------------------------------------------------------------------------------------------ head norms
class Heads:
    def __init__(self, batch, tokens, hq, hk, dim, rot, dtype, pairing="halves", kind="rms", bias=False, wide_vec=False, sections=None,
                 layout="packed", shift=0, pad=0, long=True, seed=0):
        rng = np.random.RandomState(seed + 31 * dim + tokens)
        self.dtype, self.sections, self.pairing, self.hk = dtype, sections, pairing, hk

        def heads(spread):
            if layout == "packed":
                t = made(rng, (batch, tokens, hq + 2 * hk, dim), dtype, spread, 0.1, pad, shift)
                return t[:, :, :hq], t[:, :, hq:hq + hk] if hk else None
            t = [made(rng, (batch, h, tokens, dim), dtype, spread, 0.1, pad, shift).transpose(1, 2) for h in (hq, hk)]
            return t[0], t[1] if hk else None
        (self.q, self.k), (self.dq, self.dk) = heads(1.2), heads(0.6)
        vec = F32 if wide_vec and dtype in (BF16, F16) else dtype
        norm = lambda: (kind, made(rng, (dim,), vec, 0.2, 1.0), made(rng, (dim,), vec, 0.3) if bias else None, 1e-5) if kind else None  # noqa: E731
        self.norms = [norm(), norm() if hk else None]
        self.rotate = None
        if rot:
            pairs, rows = rot // 2, tokens + 50
            angle = np.arange(rows)[:, None] * 100.0 ** (-np.arange(pairs) / pairs)
            cos, sin = (torch.from_numpy(f(angle)).to(wide(dtype)).cuda() for f in (np.cos, np.sin))
            shape = (batch, tokens) if sections is None else (len(sections), batch, tokens)
            self.positions = torch.from_numpy(rng.randint(0, rows, shape)).to(torch.int64 if long else torch.int32).cuda()
            self.rotate = (cos, sin, self.positions, pairing, sections)

    def how(self):
        return dict(q_norm=self.norms[0], k_norm=self.norms[1], rotate=self.rotate)

    def host_rotation(self):
        if self.rotate is None:
            return None
        cos, sin, pos = (host(t) for t in self.rotate[:3])
        return ref.angles(cos, sin, pos, self.sections) + (self.pairing,)

    def host_norm(self, k):
        n = self.norms[k]
        return None if n is None else (n[0], host(n[1]), host(n[2]), n[3])

    def check(self):
        u = unit(self.dtype)
        got = fo.fused_head_norm(self.q, self.k, **self.how())
        for k, x in enumerate((self.q, self.k)):
            if x is None:
                assert got[k] is None
                continue
            want, size = ref.head_norm(host(x), self.host_norm(k), self.host_rotation())
            assert got[k].dtype == self.dtype
            close(got[k], want, 64 * u * size, "qk"[k])
        grads = fo.fused_head_norm_grad(self.dq, self.dk, self.q, self.k, **self.how())
        names = set()
        for k, (d, x) in enumerate(((self.dq, self.q), (self.dk, self.k))):
            if x is None:
                continue
            n = self.norms[k]
            want = ref.head_norm_grad(host(d), host(x), self.host_norm(k), self.host_rotation())
            name = "qk"[k]
            names |= {name} | ({name + "_w"} if n else set()) | ({name + "_b"} if n and n[2] is not None else set())
            close(grads[name], want["x"][0], 64 * u * want["x"][1], "d" + name)
            vectors = x.shape[0] * x.shape[1] * x.shape[2]
            for part in "wb":
                if name + "_" + part in names:
                    assert grads[name + "_" + part].dtype == wide(self.dtype)
                    close(grads[name + "_" + part], want[part][0], (64 + vectors) * u * want[part][1], "d" + name + "_" + part)
        assert set(grads) == names


DIMS = [(1, 0), (2, 2), (3, 2), (7, 6), (16, 16), (40, 20), (63, 62), (64, 64), (72, 72), (80, 40), (96, 96), (128, 128), (128, 32), (130, 128),
        (192, 192), (200, 64), (256, 256), (257, 100), (511, 510), (512, 512)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,rot", DIMS)
def test_head_sizes(dtype, dim, rot):
    for n, (pairing, kind) in enumerate((("halves", "rms"), ("pairs", "layer"), ("halves", None), ("pairs", "rms"))):
        Heads(2, 5, 3, 1, dim, rot, dtype, pairing, kind, bias=n == 1, wide_vec=n == 3, layout=("packed", "heads first")[n % 2]).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,hq,hk", [(1, 1, 1, 0), (1, 1, 32, 8), (64, 1, 5, 5), (3, 7, 33, 1), (1, 1531, 12, 4), (2, 600, 1, 1)])
def test_head_counts(dtype, batch, tokens, hq, hk):
    Heads(batch, tokens, hq, hk, 64, 64, dtype, bias=True, long=tokens % 2 == 1).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,hq,hk,dim", [(3, 2501, 12, 4, 64), (1, 4003, 7, 3, 128), (2, 3001, 6, 0, 72), (1, 9001, 2, 1, 30)])
def test_heads_of_many_tokens(dtype, batch, tokens, hq, hk, dim):
    """Several tokens side by side in a warp, of which the last ones and those of two sequences are not as many."""
    Heads(batch, tokens, hq, hk, dim, dim, dtype, kind="layer" if dim == 72 else "rms", bias=dim == 72,
          pairing="pairs" if dim == 72 else "halves", sections=(12, 12, 12) if dim == 72 else None, layout="apart" if dim == 128 else "packed").check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 3), (4, 4), (8, 8), (2, 6)])
def test_heads_anywhere(dtype, shift, pad):
    for pairing in ("halves", "pairs"):
        Heads(2, 9, 4, 2, 96, 64, dtype, pairing, "layer", shift=shift, pad=pad).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sections", [(8, 12, 12), (16, 16), (1, 30, 0, 1), (32,), (0, 0, 32), (5, 9, 18)])
def test_head_axes(dtype, sections):
    for pairing in ("halves", "pairs"):
        Heads(2, 11, 4, 2, 80, 64, dtype, pairing, "rms", sections=sections).check()


def test_positions_outside_the_table_and_broadcast():
    c = Heads(2, 6, 3, 1, 64, 32, BF16)
    c.positions[0, 2], c.positions[1, 5], c.positions[1, 0] = -1, 56, 1 << 40
    c.check()
    q, _ = fo.fused_head_norm(c.q, **{**c.how(), "k_norm": None})
    bad = torch.isnan(q).any(-1).any(-1)
    assert bad.nonzero().tolist() == [[0, 2], [1, 0], [1, 5]] and not torch.isnan(q[..., 32:]).any()
    cos, sin = c.rotate[:2]
    shared = torch.arange(6, device="cuda")
    for q in (c.q, c.q[1]):                                  # of all sequences alike, and a batch of one without its dimension
        a, _ = fo.fused_head_norm(q, rotate=(cos, sin, shared, "halves", None))
        b, _ = fo.fused_head_norm(q, rotate=(cos, sin, shared.expand(2, 6) if q.dim() == 4 else shared, "halves", None))
        assert torch.equal(a, b)
    with_axes = torch.stack([shared, shared])
    a, _ = fo.fused_head_norm(c.q, rotate=(cos, sin, with_axes, "halves", (4, 12)))
    b, _ = fo.fused_head_norm(c.q, rotate=(cos, sin, shared, "halves", None))
    assert torch.equal(a, b)


def test_heads_in_place_and_into_a_projection():
    c = Heads(2, 37, 6, 2, 128, 128, BF16, bias=True)
    want = [t.clone() for t in fo.fused_head_norm(c.q, c.k, **c.how())]
    grads = {k: v.clone() for k, v in fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how()).items()}
    dqkv = torch.full((2, 37, 10, 128), 7.0, dtype=BF16, device="cuda")
    got = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, out_q=dqkv[:, :, :6], out_k=dqkv[:, :, 6:8], **c.how())
    assert all(torch.equal(got[k], grads[k]) for k in grads) and (dqkv[:, :, 8:] == 7.0).all()
    assert got["q"].data_ptr() == dqkv.data_ptr()
    got = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, out_q=c.dq, out_k=c.dk, **c.how())
    assert got["q"] is c.dq and all(torch.equal(got[k], grads[k]) for k in grads)
    rest = c.q._base.view(2, 37, 10, 128)[:, :, 8:].clone()
    version = c.q._version
    got = fo.fused_head_norm(c.q, c.k, out_q=c.q, out_k=c.k, **c.how())
    assert got[0] is c.q and all(torch.equal(a, b) for a, b in zip(got, want)) and c.q._version > version
    assert torch.equal(c.q._base.view(2, 37, 10, 128)[:, :, 8:], rest)


def test_head_values():
    """A head's NaN or infinity stays in it; zeros with and without eps; one tensor's gradient alone."""
    c = Heads(1, 4, 3, 2, 64, 64, F32)
    clean = fo.fused_head_norm(c.q, c.k, **c.how())[0].clone()
    c.q[0, 1, 2, 5], c.q[0, 3, 0, 63] = float("nan"), float("inf")
    got = fo.fused_head_norm(c.q, c.k, **c.how())[0]
    hit = torch.zeros(1, 4, 3, dtype=torch.bool, device="cuda")
    hit[0, 1, 2] = hit[0, 3, 0] = True
    assert torch.isnan(got[hit]).any(-1).all() and torch.equal(got[~hit], clean[~hit])
    zeros = torch.zeros(1, 5, 3, 64, device="cuda")
    assert (fo.fused_head_norm(zeros, q_norm=("rms", None, None, 1e-6))[0] == 0).all()
    assert torch.isnan(fo.fused_head_norm(zeros, q_norm=("rms", None, None, 0.0))[0]).all()
    c = Heads(2, 40, 3, 2, 64, 64, F32, bias=True)
    both = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how())
    one = fo.fused_head_norm_grad(None, c.dk, None, c.k, k_norm=c.norms[1], rotate=c.rotate)
    assert set(one) == {"k", "k_w", "k_b"} and torch.equal(one["k"], both["k"])
    empty = fo.fused_head_norm_grad(c.dq[:, :0], None, c.q[:, :0], q_norm=c.norms[0])
    assert (empty["q_w"] == 0).all() and (empty["q_b"] == 0).all() and empty["q"].numel() == 0
    assert fo.fused_head_norm(c.q[:, :, :0], c.k)[0].shape == (2, 40, 0, 64)


# ------------------------------------------------------------------------------------------------------------ recurrence
class Scan:
    def __init__(self, batch, tokens, channels, dtype, gate, decay, mix, state=True, reset=0.0, lengths=None, pad=0, shift=0, seed=0):
        rng = np.random.RandomState(seed + 13 * tokens + channels)
        one = lambda t, spread, mean=0.0: made(rng, (batch, tokens, channels), t, spread, mean, pad, shift)  # noqa: E731
        self.dtype, self.kind, self.mix = dtype, decay, mix
        self.x, self.dh, self.gate = one(dtype, 1.0), one(dtype, 0.5), one(gate, 2.0, 1.0)
        if decay == "value":
            self.gate.sigmoid_().clamp_(max=0.98)
        elif decay == "exp":
            self.gate.sigmoid_().add_(1e-3).log_().mul_(0.5).clamp_(max=-1e-3)
        self.state = made(rng, (batch, channels), wide(dtype)) if state else None
        self.dlast = made(rng, (batch, channels), wide(dtype), 0.5) if state else None
        self.reset = torch.from_numpy(rng.rand(batch, tokens) < reset).cuda() if reset else None
        self.lengths = None if lengths is None else torch.tensor(lengths, device="cuda")

    def how(self):
        return dict(decay=self.kind, mix=self.mix, state=self.state, reset=self.reset, lengths=self.lengths)

    def host_how(self):
        b, t = self.x.shape[:2]
        lengths = np.full(b, t) if self.lengths is None else np.clip(host(self.lengths), 0, t)
        return dict(kind=self.kind, mix=self.mix, state=host(self.state), reset=np.zeros((b, t), bool) if self.reset is None else host(self.reset) != 0,
                    lengths=lengths)

    def check(self):
        u = unit(self.dtype)
        h, last = fo.fused_scan(self.x, self.gate, **self.how())
        want, error, wlast, elast = ref.scan(host(self.x), host(self.gate), **self.host_how())
        assert h.dtype == self.dtype and last.dtype == wide(self.dtype)
        close(h, want, u * error, "h")
        close(last, wlast, u * elast, "last")
        got = fo.fused_scan_grad(self.dh, self.x, self.gate, h, dlast=self.dlast, **self.how())
        want = ref.scan_grad(host(self.dh), host(self.x), host(self.gate), host(h), dlast=host(self.dlast), **self.host_how())
        assert set(got) == {"x", "gate"} | ({"state"} if self.state is not None else set())
        assert got["x"].dtype == self.dtype and got["gate"].dtype == self.gate.dtype
        for k in got:
            close(got[k], want[k][0], u * want[k][1], "d" + k)
        return h, last, got


PAIRS = [(F64, F64), (F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]
MODES = [(d, m) for d in ("value", "sigmoid", "exp") for m in ("one", "rest", "root")]


@pytest.mark.parametrize("dtype,gate", PAIRS)
@pytest.mark.parametrize("decay,mix", MODES)
def test_scan_modes(dtype, gate, decay, mix):
    Scan(3, 37, 66, dtype, gate, decay, mix, reset=0.1, lengths=[37, 20, 0]).check()


@pytest.mark.parametrize("dtype,gate", PAIRS)
@pytest.mark.parametrize("tokens", [0, 1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 255, 257, 511, 513, 1030, 2049])
def test_scan_lengths(dtype, gate, tokens):
    decay, mix = MODES[(tokens + PAIRS.index((dtype, gate))) % 9]
    Scan(1, tokens, 33 if tokens % 2 else 64, dtype, gate, decay, mix, state=tokens % 4 != 3).check()


@pytest.mark.parametrize("dtype,gate", PAIRS)
@pytest.mark.parametrize("batch,channels", [(1, 1), (2, 2), (7, 31), (1, 32), (3, 63), (2, 65), (5, 130), (1, 1000), (300, 40), (40, 1001)])
def test_scan_widths(dtype, gate, batch, channels):
    Scan(batch, 19, channels, dtype, gate, "sigmoid", "rest", reset=0.05).check()
    Scan(batch, 1, channels, dtype, gate, "exp", "root").check()


@pytest.mark.parametrize("dtype,gate", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 1), (2, 2), (0, 62)])
def test_scan_anywhere(dtype, gate, shift, pad):
    Scan(2, 70, 66, dtype, gate, "sigmoid", "root", shift=shift, pad=pad).check()
    c = Scan(2, 70, 66, dtype, gate, "sigmoid", "rest")
    want = [t.clone() for t in fo.fused_scan(c.x, c.gate, **c.how())]
    c.x = c.x.transpose(0, 1).contiguous().transpose(0, 1)  # tokens before the batch
    got = fo.fused_scan(c.x, c.gate, **c.how())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_masks(dtype):
    """Lengths beyond both ends, 32-bit lengths, bytes as marks, NaN and infinities where nothing is looked at, resets everywhere."""
    c = Scan(5, 90, 64, dtype, dtype, "sigmoid", "rest", reset=0.1, lengths=[90, 0, -3, 1000, 41])
    h, last, got = c.check()
    c.lengths = c.lengths.int()
    c.reset = c.reset.byte() * 5
    for t, bad in ((c.x, float("nan")), (c.gate, float("inf")), (c.dh, float("-inf"))):
        t[4, 41:] = bad
        t[1] = bad
    h2, last2, got2 = c.check()
    assert torch.equal(h, h2) and torch.equal(last, last2) and all(torch.equal(got[k], got2[k]) for k in got)
    assert (h[4, 41:] == 0).all() and torch.equal(last[1], c.state[1]) and torch.equal(got["state"][1], c.dlast[1])
    c = Scan(2, 50, 64, dtype, dtype, "exp", "one")
    c.reset = torch.ones(2, 50, dtype=torch.bool, device="cuda")
    c.state.fill_(float("nan"))                              # dropped before it is used
    h, last, got = c.check()
    assert torch.equal(h, c.x) and (got["state"] == 0).all() and (got["gate"] == 0).all()
    c = Scan(1, 130, 64, dtype, dtype, "sigmoid", "rest")
    c.x[0, 20] = float("inf")
    c.reset = torch.zeros(1, 130, dtype=torch.bool, device="cuda")
    c.reset[0, 100] = True
    h, last = fo.fused_scan(c.x, c.gate, **c.how())
    assert not torch.isfinite(h[0, 20:100]).any() and torch.isfinite(h[0, :20]).all() and torch.isfinite(h[0, 100:]).all()


@pytest.mark.parametrize("dtype,gate", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_scan_step_by_step(dtype, gate):
    """Tokens one at a time, states handed on in place, are the sequence; so are its halves."""
    c = Scan(3, 24, 70, dtype, gate, "sigmoid", "root")
    u = unit(dtype)
    want, error, wlast, elast = ref.scan(host(c.x), host(c.gate), **c.host_how())
    for cuts in (list(range(25)), [0, 11, 24], [0, 24]):
        state, out = c.state.clone(), torch.full_like(c.x, 9.0)
        for a, b in zip(cuts, cuts[1:]):
            h, last = fo.fused_scan(c.x[:, a:b], c.gate[:, a:b], c.kind, c.mix, state, out=out[:, a:b], out_state=state)
            assert last is state and h.data_ptr() == out[:, a:b].data_ptr()
        close(out, want, u * error, "h")
        close(state, wlast, u * elast, "last")
    one = fo.fused_scan(c.x[0], c.gate[0], c.kind, c.mix, c.state[0])       # without a batch
    all_ = fo.fused_scan(c.x, c.gate, c.kind, c.mix, c.state)
    assert torch.equal(one[0], all_[0][0]) and torch.equal(one[1], all_[1][0])
    x = c.x.clone()
    assert torch.equal(fo.fused_scan(x, c.gate, c.kind, c.mix, c.state, out=x)[0], all_[0])


def test_scan_long_memory():
    """Decays next to 1 over a long sequence: the error of a decay is one rounding, however often it is applied."""
    for gate, decay in ((9.0, "sigmoid"), (-1e-4, "exp"), (0.9999, "value")):
        c = Scan(1, 30000, 64, BF16, F32, decay, "rest")
        c.gate.fill_(gate)
        c.check()


@pytest.mark.parametrize("dtype,gate", PAIRS)
@pytest.mark.parametrize("tokens,batch,channels", [(8192, 1, 33), (8200, 3, 66), (9001, 2, 200), (8193, 4, 1)])
def test_scan_in_chunks(dtype, gate, tokens, batch, channels):
    """Sequences that are long for their channels: ends in the first, a middle and the last chunk, at a border and nowhere, chunks with
    resets and without."""
    decay, mix = MODES[(tokens + PAIRS.index((dtype, gate))) % 9]
    lengths = [tokens - 3, 4096, 700, 0][:batch] if batch > 1 else None
    Scan(batch, tokens, channels, dtype, gate, decay, mix, reset=0.0004, lengths=lengths).check()
    Scan(batch, tokens, channels, dtype, gate, "sigmoid", "rest", state=False, lengths=lengths, shift=1, pad=3).check()


def test_scan_in_chunks_and_in_one():
    """In place, without gradients of one result, and marks at the borders of all segments."""
    c = Scan(2, 12288, 64, BF16, BF16, "sigmoid", "rest")
    h, last = fo.fused_scan(c.x, c.gate, **c.how())
    x, state = c.x.clone(), c.state.clone()
    got = fo.fused_scan(x, c.gate, c.kind, c.mix, state, out=x, out_state=state)
    assert torch.equal(got[0], h) and torch.equal(got[1], last) and got[0].data_ptr() == x.data_ptr()
    zero = torch.zeros_like(c.dh)
    a = fo.fused_scan_grad(None, c.x, c.gate, h, dlast=c.dlast, **c.how())
    b = fo.fused_scan_grad(zero, c.x, c.gate, h, dlast=c.dlast, **c.how())
    assert all(torch.equal(a[k], b[k]) for k in b)
    c.reset = torch.zeros(2, 12288, dtype=torch.bool, device="cuda")
    c.reset[0, ::64] = True
    c.reset[1, 63::64] = True
    c.check()


def test_scan_missing_gradients():
    c = Scan(2, 33, 64, BF16, BF16, "sigmoid", "one")
    h, _ = fo.fused_scan(c.x, c.gate, **c.how())
    zero = torch.zeros_like(c.dh)
    a = fo.fused_scan_grad(None, None, c.gate, h, dlast=c.dlast, **c.how())
    b = fo.fused_scan_grad(zero, c.x, c.gate, h, dlast=c.dlast, **c.how())
    assert all(torch.equal(a[k], b[k]) for k in b)
    a = fo.fused_scan_grad(c.dh, c.x, c.gate, h, **c.how())
    b = fo.fused_scan_grad(c.dh, c.x, c.gate, h, dlast=torch.zeros_like(c.dlast), **c.how())
    assert all(torch.equal(a[k], b[k]) for k in b)


# ------------------------------------------------------------------------------------------------------------ distillation
class Distill:
    def __init__(self, rows, vocab, top, dtype, tail, temperature=1.0, values=None, long=True, pad=0, shift=0, seed=0):
        rng = np.random.RandomState(seed + vocab + 7 * rows)
        self.temperature, self.dtype = temperature, dtype
        self.logits = made(rng, (rows, vocab), dtype, 2.5, 0.3, pad, shift)
        teacher = host(self.logits) * 1.1 + rng.randn(rows, vocab)
        ids = np.argsort(-teacher, axis=1, kind="stable")[:, :top]
        self.ids = torch.from_numpy(ids.copy()).to(torch.int64 if long else torch.int32).cuda()
        self.values = torch.from_numpy(np.take_along_axis(teacher, ids, 1)).to(values or dtype).cuda()
        self.tail = None
        if tail:
            np.put_along_axis(teacher, ids, host(self.values), 1)
            t = teacher / temperature
            lse = np.log(np.exp(t - t.max(1, keepdims=True)).sum(1)) + t.max(1) if vocab else np.zeros(rows)
            self.tail = torch.from_numpy(lse).to(wide(dtype)).cuda()
        self.dloss = torch.from_numpy(rng.rand(rows) + 0.5).to(wide(dtype)).cuda()

    def args(self):
        return self.logits, self.ids, self.values

    def how(self):
        return dict(tail=self.tail, temperature=self.temperature)

    def check(self):
        rows, vocab = self.logits.shape
        u = unit(self.dtype)
        values = host(self.values)
        want, stats, dz, q = ref.distill(host(self.logits), host(self.ids), values, host(self.tail), self.temperature)
        weight = host(self.dloss)[:, None]
        # additions of a thread: its share of the row, never more than 2048 values
        delta = u * (2048 + 32)
        with np.errstate(invalid="ignore"):
            z = host(self.logits)
            far = np.where(np.isfinite(z), np.abs(z - stats[0][:, None]) / self.temperature, 0.0)
            size = np.abs(want) + np.where(np.isfinite(values), np.abs(values), 0.0).max(1, initial=0.0) / self.temperature + 100.0
            eloss = 1.1 * delta + 2.0 ** -50 * size
            ratio = np.abs(1.0 - stats[2]) + 1e-12
            eq = q * (delta + u * (16 + 2 * far))
            edz = weight / self.temperature * (eq * np.abs(stats[2])[:, None] + 2 * eq + q * (ratio * 3 * delta + 2 * u)[:, None] + 2.0 ** -40)
        loss, got = fo.fused_distill(*self.args(), stats=True, **self.how())
        assert loss.dtype == wide(self.dtype) and got.shape == (3, rows)
        close(loss, want, eloss, "loss")
        close(got[0], stats[0], 0.0, "largest")
        close(got[1], stats[1], delta * stats[1], "sum")
        close(got[2], stats[2], 3 * delta * ratio + 2 * u, "factor")
        one, step = fo.fused_distill_step(self.dloss, *self.args(), **self.how())
        assert torch.equal(one, loss) or np.allclose(host(one), host(loss), rtol=0, atol=0, equal_nan=True)
        close(step, weight * dz, edz, "dz of the step")
        close(fo.fused_distill_grad(self.dloss, *self.args(), got, **self.how()), weight * dz, edz, "dz")
        return loss, got, step


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 15, 17, 31, 64, 100, 129, 255, 1000, 1025, 4099, 8192, 20001, 32000, 50257, 128001, 180000])
def test_distill_sizes(dtype, vocab):
    for k, tail in enumerate((True, False)):
        Distill(3, vocab, min(vocab, (5, 64)[k]), dtype, tail, (1.0, 2.5)[k], long=k == 0,
                values=F32 if dtype in (BF16, F16) and k else None).check()


@pytest.mark.parametrize("dtype,vocab", [(BF16, 120001), (F16, 131072), (F32, 70003), (F64, 30011)])
def test_distill_long_rows(dtype, vocab):
    """More rows than SMs, each of more pieces than a thread keeps on their way."""
    Distill(160, vocab, 33, dtype, True, pad=vocab % 2, shift=vocab % 8).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 1), (3, 5), (8, 8)])
def test_distill_anywhere(dtype, shift, pad):
    for vocab in (50, 777, 40003):
        c = Distill(4, vocab, 9, dtype, True, 0.7, shift=shift, pad=pad)
        _, stats, step = c.check()
        # into rows that lie otherwise, and into the logits themselves; what is between the rows stays
        wide_out = torch.full((4, vocab + 3), 7.0, dtype=dtype, device="cuda")
        _, got = fo.fused_distill_step(c.dloss, *c.args(), out=wide_out[:, 2:vocab + 2], **c.how())
        assert torch.equal(got, step) and (wide_out[:, :2] == 7.0).all() and (wide_out[:, vocab + 2:] == 7.0).all()
        want = fo.fused_distill_grad(c.dloss, *c.args(), stats, **c.how())
        wide_out.fill_(7.0)
        got = fo.fused_distill_grad(c.dloss, *c.args(), stats, out=wide_out[:, 1:vocab + 1], **c.how())
        assert torch.equal(got, want) and (wide_out[:, :1] == 7.0).all() and (wide_out[:, vocab + 1:] == 7.0).all()
        keep = c.logits.clone()
        got = fo.fused_distill_grad(c.dloss, *c.args(), stats, out=c.logits, **c.how())
        assert got is c.logits and torch.equal(got, want)
        c.logits.copy_(keep)
        assert torch.equal(fo.fused_distill_step(c.dloss, *c.args(), out=c.logits, **c.how())[1], step)


@pytest.mark.parametrize("dtype", [F64, F32, BF16])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_entries(dtype, tail):
    """Entries that are none, the same place twice, more entries than a CTA's threads, all of the vocabulary, none at all."""
    c = Distill(6, 3000, 40, dtype, tail)
    c.ids[0, 5:] = -1
    c.ids[1] = -1
    c.ids[2, 7] = c.ids[2, 3]
    c.ids[2, 9] = c.ids[2, 3]
    c.ids[3, ::2] = -(1 << 20)
    c.values[4, 10:] = float("-inf")
    loss, _, dz = c.check()
    if not tail:
        assert loss[1] == 0 and (dz[1] == 0).all()
    Distill(2, 1500, 1024, dtype, tail).check()
    c = Distill(3, 200, 0, dtype, tail)
    c.check()
    if tail:
        c = Distill(3, 64, 64, dtype, tail)
        c.tail -= 0.05                                       # shares that add up to more than 1: nothing is left
        c.check()
    else:
        Distill(3, 64, 64, dtype, tail).check()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_distill_masked_logits(dtype):
    """Minus infinity and the type's lowest value in the logits; a NaN, an infinity and an id that is too large stay in their rows."""
    c = Distill(7, 2000, 8, dtype, False)
    free = torch.ones(7, 2000, dtype=torch.bool, device="cuda").scatter_(1, c.ids, False)
    c.logits[1][free[1]] = float("-inf")
    c.logits[2][free[2]] = torch.finfo(dtype).min
    c.logits[3, :1000][free[3, :1000]] = float("-inf")
    loss, stats, dz = c.check()
    assert torch.isfinite(loss).all() and torch.isfinite(dz).all()
    clean = dz.clone()
    c.logits[4, 77] = float("nan")
    c.logits[5, 9] = float("inf")
    c.ids[6, 2] = 2000
    loss, dz = fo.fused_distill_step(c.dloss, *c.args(), **c.how())
    assert torch.isnan(loss[4:]).all() and torch.isnan(dz[4:]).any(1).all() and torch.isnan(dz[6]).all()
    assert torch.equal(dz[:4], clean[:4])
    loss, stats = fo.fused_distill(*c.args(), stats=True, **c.how())
    dz = fo.fused_distill_grad(c.dloss, *c.args(), stats, **c.how())
    assert torch.isnan(loss[4:]).all() and torch.isnan(dz[6]).all() and torch.isfinite(dz[:4]).all()
    # rows that do not count are not looked at
    c.dloss[4:] = 0
    for loss, dz in (fo.fused_distill_step(c.dloss, *c.args(), **c.how()),
                     (torch.zeros(7), fo.fused_distill_grad(c.dloss, *c.args(), stats, **c.how()))):
        assert (loss[4:] == 0).all() and (dz[4:] == 0).all() and torch.isfinite(dz[:4]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_entries_that_are_all_there_is(dtype):
    """With a tail and nothing outside the entries, what rounding leaves of the teacher's other shares is not compared with nothing."""
    for vocab in (1, 2, 17, 300):
        c = Distill(400, vocab, vocab, F32 if dtype == F64 else dtype, True, temperature=0.7)
        loss, _, dz = c.check()
        assert torch.isfinite(loss).all() and torch.isfinite(dz).all()
    c = Distill(300, 1000, 1000, F32 if dtype == F64 else dtype, True)
    c.ids, c.values = c.ids[:, :12].contiguous(), c.values[:, :12].contiguous()
    c.tail = c.values.to(c.tail.dtype).logsumexp(1)
    free = torch.ones(300, 1000, dtype=torch.bool, device="cuda").scatter_(1, c.ids, False)
    for bad in (float("-inf"), torch.finfo(c.dtype).min):
        c.logits[free] = bad
        loss, _, dz = c.check()
        assert torch.isfinite(loss).all() and torch.isfinite(dz).all()
    c.tail += 0.1                                            # a tenth of the teacher's shares lies where the student's are zero
    assert torch.isinf(fo.fused_distill(*c.args(), **c.how())[0]).all()
    if dtype == F64:                                         # in 64 bits the sums' last bits are the bound's too
        c = Distill(500, 200, 200, F64, True)
        loss, stats = fo.fused_distill(*c.args(), stats=True, **c.how())
        want = ref.distill(host(c.logits), host(c.ids), host(c.values), host(c.tail), 1.0)[0]
        # 200 additions in each of four sums of shares and probabilities, times logarithms below 32
        assert np.abs(host(loss) - want).max() <= 4 * 200 * 32 * 2.0 ** -53
        assert torch.isfinite(fo.fused_distill_grad(None, *c.args(), stats, **c.how())).all()


def test_distill_is_cross_entropy_for_one_entry():
    rng = np.random.RandomState(3)
    z = made(rng, (50, 1003), F32, 3.0)
    label = torch.from_numpy(rng.randint(0, 1003, (50, 1))).cuda()
    loss, dz = fo.fused_distill_step(None, z, label, torch.zeros(50, 1, device="cuda"))
    zd = z.double().requires_grad_()
    want = torch.nn.functional.cross_entropy(zd, label[:, 0], reduction="none")
    want.sum().backward()
    assert torch.allclose(loss.double(), want, rtol=1e-6, atol=1e-6) and torch.allclose(dz.double(), zd.grad, rtol=1e-5, atol=1e-7)


# ------------------------------------------------------------------------------------------- derivatives by differences
def test_gradients_against_differences():
    """In float64, central differences of the framework's own forward calls: error about step^2 and 2^-53 / step."""
    rng = np.random.RandomState(11)
    step, rel = 1e-5, 1e-7

    def compare(f, t, grad, what, places=12):
        for _ in range(places):
            i = tuple(rng.randint(0, n) for n in t.shape)
            keep = t[i].item()
            t[i] = keep + step
            up = f()
            t[i] = keep - step
            down = f()
            t[i] = keep
            want = (up - down) / (2 * step)
            assert abs(want - grad[i].item()) <= rel * (1.0 + abs(want)), (what, i, want, grad[i].item())

    h = Heads(2, 3, 4, 2, 24, 16, F64, "pairs", "layer", bias=True, sections=(3, 5))
    total = lambda: sum((a * b).sum().item() for a, b in zip(fo.fused_head_norm(h.q, h.k, **h.how()), (h.dq, h.dk)))  # noqa: E731
    g = fo.fused_head_norm_grad(h.dq, h.dk, h.q, h.k, **h.how())
    for name, t in (("q", h.q), ("k", h.k), ("q_w", h.norms[0][1]), ("q_b", h.norms[0][2]), ("k_w", h.norms[1][1]), ("k_b", h.norms[1][2])):
        compare(total, t, g[name], name)
    for decay, mix in MODES:
        s = Scan(2, 20, 6, F64, F64, decay, mix, reset=0.1, lengths=[20, 13])
        first, _ = fo.fused_scan(s.x, s.gate, **s.how())
        g = fo.fused_scan_grad(s.dh, s.x, s.gate, first, dlast=s.dlast, **s.how())

        def total():
            y, last = fo.fused_scan(s.x, s.gate, **s.how())
            return (y * s.dh).sum().item() + (last * s.dlast).sum().item()
        for name, t in (("x", s.x), ("gate", s.gate), ("state", s.state)):
            compare(total, t, g[name], (decay, mix, name))
    for tail in (False, True):
        d = Distill(3, 40, 6, F64, tail, 1.7)
        total = lambda: (fo.fused_distill(*d.args(), **d.how())[0] * d.dloss).sum().item()  # noqa: E731
        compare(total, d.logits, fo.fused_distill_step(d.dloss, *d.args(), **d.how())[1], ("logits", tail), 30)
