"""Calls of the head norms, the recurrence and the distillation loss at the edges of what they allow.  Tolerances as in test_gpu_lm.py
where nothing else is said."""
import numpy as np
import pytest
import torch

import paper_1801_00829_b200 as fo
from test_gpu_lm import BF16, F16, F32, F64, PAIRS, TYPES, Distill, Heads, close, host, ref, unit, wide

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------ head norms
def many_tokens(dtype, pairing):
    """A warp's groups take a token each, and the last warp has fewer tokens than groups."""
    return Heads(1, 4003, 7, 3, 64, 48, dtype, pairing, "rms", bias=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", ["halves", "pairs"])
def test_heads_of_tables_without_rows(dtype, pairing):
    """Every position is outside: what is turned is NaN, the rest as without a rotation."""
    c = many_tokens(dtype, pairing)
    cos, sin = c.rotate[:2]
    c.rotate = (cos[:0], sin[:0]) + c.rotate[2:]
    c.check()
    assert torch.isnan(fo.fused_head_norm(c.q, c.k, **c.how())[0][..., :48]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairing", ["halves", "pairs"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_heads_beside_a_table_row_that_no_token_uses(dtype, pairing, bad):
    c = many_tokens(dtype, pairing)
    c.positions.clamp_(min=1)
    want = list(fo.fused_head_norm(c.q, c.k, **c.how()))
    grads = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how())
    for t in c.rotate[:2]:
        t[0] = bad
    got = fo.fused_head_norm(c.q, c.k, **c.how())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how())
    assert all(torch.equal(got[k], grads[k]) for k in grads)


@pytest.mark.parametrize("tokens_first", [True, False])
def test_as_many_vectors_as_there_may_be(tokens_first):
    count = 2 ** 31 - 1
    x = torch.empty(count, dtype=BF16, device="cuda").bernoulli_().mul_(2.0).sub_(1.0)
    x = x.view(count, 1, 1) if tokens_first else x.view(1, count, 1)
    norm = ("rms", torch.full((1,), 1.5, dtype=BF16, device="cuda"), None, 0.0)
    y, _ = fo.fused_head_norm(x, q_norm=norm)
    assert torch.equal(y, x * 1.5)
    got = fo.fused_head_norm_grad(y, None, x, q_norm=norm, out_q=y)
    # one value is its own norm: no gradient but what 1 / sqrt(x^2) is off by, two units; the sums of 1.5 in lines of 2^16 and then lines
    assert got["q"].abs().max() <= 1.5 * 1.5 * 8 * 2.0 ** -24 and abs(got["q_w"].item() / (1.5 * count) - 1.0) <= 2.0 ** -8


# ------------------------------------------------------------------------------------------------------------ recurrence
@pytest.mark.parametrize("dtype,gate", PAIRS)
@pytest.mark.parametrize("mix", ["one", "rest", "root"])
@pytest.mark.parametrize("tokens", [1, 3, 40, 700, 9001])
def test_small_decays_are_right_relative_to_themselves(dtype, gate, mix, tokens):
    """Every other token adds nothing, so that all of its h is a small decay times the h before it."""
    rng = np.random.RandomState(tokens)
    g = torch.from_numpy(rng.uniform(-18.0, -6.0, (2, tokens, 70))).to(gate).cuda()
    x = torch.from_numpy(rng.uniform(500.0, 1000.0, (2, tokens, 70))).to(dtype).cuda()
    x[:, ::2] = 0
    state = torch.from_numpy(rng.uniform(500.0, 1000.0, (2, 70))).to(wide(dtype)).cuda()
    h, last = fo.fused_scan(x, g, "sigmoid", mix, state)
    gd = host(g)
    a, rest = ref.decay(gd, "sigmoid")
    m = ref.mixed(a, rest, mix) * host(x)
    want, carry = np.zeros_like(gd), host(state)
    for t in range(tokens):
        want[:, t] = carry = a[:, t] * carry + m[:, t]
    # a is off by 24 + 4 |gate| units of itself (exponent, exponential, reciprocal, product), and so is the h that it is all of; that
    # before it by the 24 + 4 |gate| of m(a), and two more products and sums
    relative = 2 * (24 + 4 * np.abs(gd) + 8) * unit(dtype)
    close(h, want, np.abs(want) * relative, "h")
    if tokens % 2:
        close(last, carry, np.abs(carry) * relative[:, -1], "last")


def test_as_many_channels_as_there_may_be():
    """2^28 channels in 64 bits are 2^31 bytes a row."""
    channels = 1 << 28
    x, gate = torch.rand(channels, dtype=F64, device="cuda"), torch.rand(channels, dtype=F64, device="cuda")
    h, last = fo.fused_scan(x.expand(5, -1), gate.expand(5, -1), "value", "rest")
    parts = (slice(0, 4096), slice(channels // 2 - 64, channels // 2 + 64), slice(channels - 4096, channels))
    for part in parts:
        want = torch.zeros_like(x[part])
        for t in range(5):
            want = gate[part] * want + (1.0 - gate[part]) * x[part]
            assert (h[t, part] - want).abs().max() <= 16 * 2.0 ** -53
        assert torch.equal(last[part], h[4, part])
    del last
    got = fo.fused_scan_grad(x.expand(5, -1), None, gate.expand(5, -1), h, "value", "one")
    for part in parts:
        want = torch.zeros_like(x[part])
        for t in range(4, -1, -1):
            want = x[part] + gate[part] * want
            assert (got["x"][t, part] - want).abs().max() <= 32 * 2.0 ** -53
            before = h[t - 1, part] if t else 0.0
            assert (got["gate"][t, part] - want * before).abs().max() <= 64 * 2.0 ** -53


def test_as_many_tokens_as_there_may_be():
    """2^30 tokens, in chunks; far back nothing is left of a state, so that windows of the sequence can be looked at by themselves."""
    count, window, lead = 1 << 30, 300, 200                  # a is at most 0.73: 0.73^200 is 2^-90
    x = torch.empty(count, 1, dtype=BF16, device="cuda").uniform_(-1.0, 1.0)
    gate = torch.empty(count, 1, dtype=BF16, device="cuda").uniform_(-1.0, 1.0)
    reset = torch.zeros(count, dtype=torch.bool, device="cuda")
    places = [0, 12345, (1 << 29) - 150, count - window - lead]
    for first in places:
        reset[first + lead + 77] = True
    state = torch.full((1,), 3.0, device="cuda")
    h, last = fo.fused_scan(x, gate, "sigmoid", "rest", state, reset)
    got = fo.fused_scan_grad(x, x, gate, h, "sigmoid", "rest", state, reset, dlast=state)
    assert last.item() == pytest.approx(h[-1].item(), rel=2.0 ** -8, abs=2.0 ** -126)
    for first in places:
        part = slice(first, first + window + lead)
        a = torch.sigmoid(gate[part, 0].double())
        drop, xd, hd = reset[part], x[part, 0].double(), h[part, 0].double()
        want, s = torch.zeros_like(a), state[0].double() if first == 0 else torch.zeros((), dtype=F64, device="cuda")
        for t in range(window + lead):
            s = (0.0 if drop[t] else a[t] * s) + (1.0 - a[t]) * xd[t]
            want[t] = s
        at = slice(0 if first == 0 else lead, window + lead)
        # sums of numbers below 1 (3 with the state) in 32 bits, at most 4 of them in effect, and one rounding
        assert ((want - hd)[at].abs() <= 2.0 ** -8 * want[at].abs() + 64 * 3 * 2.0 ** -24).all(), first
        through, dx, dg = torch.zeros_like(s), torch.zeros_like(a), torch.zeros_like(a)
        if first == places[-1]:
            through = state[0].double()
        for t in reversed(range(window + lead)):
            lam = xd[t] + through
            before = 0.0 if drop[t] else (hd[t - 1] if t else state[0].double())
            dx[t], dg[t] = (1.0 - a[t]) * lam, a[t] * (1.0 - a[t]) * lam * (before - xd[t])
            through = torch.zeros_like(s) if drop[t] else a[t] * lam
        at = slice(1 if first else 0, window + lead if first == places[-1] else window)
        for name, v in (("x", dx), ("gate", dg)):
            assert ((v - got[name][part, 0].double())[at].abs() <= 2.0 ** -8 * v[at].abs() + 64 * 12 * 2.0 ** -24).all(), (name, first)
    with pytest.raises(fo.FusedOpsError):
        fo.fused_scan(x[:1].expand(count + 1, 1), gate[:1].expand(count + 1, 1), lengths=torch.zeros(1, dtype=torch.int64, device="cuda"), out=None)


def test_as_many_sequences_as_there_may_be():
    count = 2 ** 31 - 1
    x = torch.empty(count, 1, 1, dtype=BF16, device="cuda").bernoulli_()
    h, last = fo.fused_scan(x, x, "value", "one")
    assert torch.equal(h, x) and torch.equal(last, x[:, 0].float())
    _, again = fo.fused_scan(x, x, "value", "one", last, out=h, out_state=last)
    assert again is last and torch.equal(h, x * 2.0) and torch.equal(last[-4096:], h[-4096:, 0].float())


# ------------------------------------------------------------------------------------------------------------ distillation
def compare(c):
    """Loss, statistics and both gradients with the oracle.

    As in test_gpu_lm.py, and: `top` shares are added up in 64 bits by the kernel and by the oracle, and their sum, and what it leaves of
    1, is off by `top` additions and 32 units of a share in each (float64's other errors are no larger).  The exponent of an exponential
    outside the entries is a distance to the largest logit and, where a student is sure, the logarithm of P / Q (at most 20 beyond the
    distance), each rounded up to three times by the units of their sizes."""
    top, t, u, values = c.ids.shape[1], c.temperature, unit(c.dtype), host(c.values)
    want, stats, dz, q = ref.distill(host(c.logits), host(c.ids), values, host(c.tail), t)
    weight, z = host(c.dloss)[:, None], host(c.logits)
    delta, off = u * (2048 + 32), 2 * (top + 32) * 2.0 ** -53
    with np.errstate(invalid="ignore"):
        far = np.where(np.isfinite(z), np.abs(z - stats[0][:, None]) / t, 0.0)
    ids = host(c.ids)
    outside = np.ones(z.shape, dtype=bool)
    for r, row in enumerate(ids):
        outside[r, row[row >= 0]] = False
    elsewhere = np.where(outside, q, 0.0).sum(1)             # Q
    p = np.zeros(0) if c.tail is None else np.where(ids >= 0, np.exp(values / t - host(c.tail)[:, None]), 0.0).sum(1)
    rest = np.zeros(len(z)) if c.tail is None else np.where(elsewhere > 0, np.maximum(1.0 - p, 0.0), 0.0)       # P
    with np.errstate(divide="ignore", invalid="ignore"):
        ratio = np.where(rest > 0, rest / elsewhere, 0.0)
        # (also where one of the two has nothing left and the other a last bit)
        eratio = np.where((elsewhere > 0) & (c.tail is not None), 3 * delta * ratio + off / elsewhere, 0.0)
    size = np.abs(want) + np.where(np.isfinite(values), np.abs(values), 0.0).max(1, initial=0.0) / t + 100.0
    loss, kept = fo.fused_distill(*c.args(), stats=True, **c.how())
    close(loss, want, 1.1 * delta + 2.0 ** -50 * size + off * (np.log(ratio + 1.0) + 40.0), "loss")
    close(kept[0], stats[0], 0.0, "largest")
    sure = ratio > 2.0 ** 60
    close(kept[1], np.where(sure, -stats[1], stats[1]), delta * stats[1], "sum")
    log = np.log(np.maximum(ratio, 1.0))
    close(kept[2], np.where(sure, log, stats[2]), np.where(sure, eratio / np.maximum(ratio, 1.0) + 2 * u * log, eratio + 2 * u + off), "factor")
    relative = delta + u * (16 + 6 * (far + 20.0))
    edz = (q * (2.0 + np.where(outside, ratio[:, None], 0.0)) * relative + np.where(outside, q * eratio[:, None], 0.0) + 2.0 ** -44) / t
    one, step = fo.fused_distill_step(c.dloss, *c.args(), **c.how())
    assert torch.equal(one, loss)
    close(step, weight * dz, weight * edz, "dz of the step")
    close(fo.fused_distill_grad(c.dloss, *c.args(), kept, **c.how()), weight * dz, weight * edz, "dz")
    return loss, kept, step


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,vocab", [(9, 32000), (9, 700), (200, 700), (200, 5000), (200, 100)])
def test_distill_minus_infinity_at_entries(dtype, tail, rows, vocab):
    """A vocabulary that is masked for teacher and student alike, and masked logits at entries with shares and without."""
    c = Distill(rows, vocab, 64, dtype, tail)
    inf = float("inf")
    for r in (0, 1, rows - 1):                               # five are allowed
        keep = c.logits[r, c.ids[r, :5]].clone()
        c.logits[r] = -inf
        c.logits[r, c.ids[r, :5]] = keep
        c.values[r, 5:] = -inf
        if tail:
            c.tail[r] = c.values[r, :5].to(c.tail.dtype).logsumexp(0)
    for r, (low, high) in ((2, (32, 64)), (3, (0, 32)), (4, (40, 41)), (5, (1, 64))):
        c.logits[r, c.ids[r, low:high]] = -inf
        c.values[r, low:high] = -inf
    c.logits[6, c.ids[6, 7]] = -inf                          # has a share: the loss is infinite, the gradient is not
    c.logits[7, c.ids[7]] = -inf
    loss, stats, dz = compare(c)
    assert torch.isinf(loss[6:8]).all() and torch.isfinite(loss[:6]).all() and torch.isfinite(dz).all() and not torch.isnan(stats).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(5, 50257), (300, 777)])
def test_distill_a_masked_label(dtype, rows, vocab):
    c = Distill(rows, vocab, 1, dtype, False)
    c.logits[1, c.ids[1, 0]] = -float("inf")
    loss, _, dz = compare(c)
    assert torch.isinf(loss[1]) and torch.isfinite(loss[2:]).all() and torch.isfinite(dz).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temperature", [1.0, 0.5])
@pytest.mark.parametrize("rows,vocab,top", [(6, 3000, 12), (300, 60, 5), (4, 40003, 70)])
def test_distill_a_student_that_is_sure(dtype, temperature, rows, vocab, top):
    """The teacher leaves a share outside the entries, where the student has next to nothing: down to exp(-680) (with the clamped logits' 8 or 16
    more at both temperatures; beyond exp(-708) the oracle's own numbers lose bits)."""
    rng = np.random.RandomState(vocab)
    for gap in (20.0, 41.0, 60.0, 86.0, 89.0, 105.0, 200.0, 400.0, 660.0):
        c = Distill(rows, vocab, top, dtype, True, temperature)
        c.logits.clamp_(-4.0, 4.0)
        c.logits.scatter_add_(1, c.ids, torch.full(c.ids.shape, gap * temperature, dtype=dtype, device="cuda"))
        free = torch.ones(rows, vocab, dtype=torch.bool, device="cuda").scatter_(1, c.ids, False)
        c.logits[0][free[0].logical_and(torch.arange(vocab, device="cuda") % 3 == 0)] = -float("inf")
        left = torch.from_numpy(rng.choice([1e-6, 0.01, 0.03, 0.04, 0.2, 0.9], rows)).cuda()
        c.tail = ((c.values.double() / temperature).logsumexp(1) - torch.log1p(-left)).to(wide(dtype))
        loss, _, dz = compare(c)
        assert torch.isfinite(loss).all() and torch.isfinite(dz).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(6, 3000), (300, 500)])
def test_distill_a_student_with_almost_all_elsewhere(dtype, rows, vocab):
    """The student's share outside is 1 but for rounding, the teacher's is small: it counts all the same, in both gradients."""
    for low in (-6.0, -8.0, -10.0, -12.0, -30.0):
        c = Distill(rows, vocab, 6, dtype, True)
        c.logits.clamp_(-1.0, 1.0)
        c.logits.scatter_(1, c.ids, low)
        c.values[:, 3:] = -float("inf")                      # no share: the gradient there is q S
        c.tail = (c.values.double().logsumexp(1) - np.log(1.0 - 0.03)).to(wide(dtype))
        compare(c)


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_temperatures_out_of_all_bounds(dtype):
    """Beyond the range of 32 bits: next to no difference between the logits, but for masked ones, and none that is not infinite."""
    z = torch.tensor([[3.0, 1.0, -float("inf"), 2.0, -1.0] * 60, [0.0, 4.0, 1.0, -float("inf"), 2.0] * 60], dtype=dtype, device="cuda")
    z[1, 1] = 5.0
    ids, values = torch.tensor([[0, 1], [1, 2]], device="cuda"), torch.zeros(2, 2, dtype=dtype, device="cuda")
    for temperature in (1e37, 1e39, 1e44, 1e46, 1e120, 1e299):
        loss, stats = fo.fused_distill(z, ids, values, temperature=temperature, stats=True)
        # the shares are halves, q is 1 / 240
        assert (loss.double() - np.log(120.0)).abs().max() <= 2.0 ** -20 and (stats[1] == 240).all()
        for dz in (fo.fused_distill_step(None, z, ids, values, temperature=temperature)[1], fo.fused_distill_grad(None, z, ids, values, stats, temperature=temperature)):
            assert torch.isfinite(dz).all() and dz.abs().max() <= 1e-36
    for temperature in (1e-37, 1e-39, 1e-44, 1e-120, 1e-299):
        one = torch.tensor([[1], [1]], device="cuda")
        loss, stats = fo.fused_distill(z, one, values[:, :1], temperature=temperature, stats=True)
        assert stats[:, 1].tolist() == [5.0, 1.0, 1.0] and loss[1] == 0 and loss[0] > 1e37
        for dz in (fo.fused_distill_step(None, z, one, values[:, :1], temperature=temperature)[1],
                   fo.fused_distill_grad(None, z, one, values[:, :1], stats, temperature=temperature)):
            assert (dz[1] == 0).all() and not torch.isnan(dz).any()
    for temperature in (0.0, -1.0, float("nan"), float("inf"), 1e301, 1e-301):
        with pytest.raises(fo.FusedOpsError):
            fo.fused_distill(z, ids, values, temperature=temperature)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,shift", [(1 << 20, 0), ((1 << 20) - 3, 1)])
def test_distill_as_many_logits_and_entries_as_there_may_be(dtype, vocab, shift):
    for rows, tail in ((1, True), (3, False)):
        compare(Distill(rows, vocab, 1024, dtype, tail, 0.7, shift=shift))
