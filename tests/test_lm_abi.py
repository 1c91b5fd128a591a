"""Refusals of the head norms, the recurrence and the distillation loss: found on the host, before anything is launched (the first
tests need no GPU)."""
import math
import struct

import pytest
import torch

import paper_1801_00829_b200 as fo

F64, F32, BF16, F16, I32, I64 = 0, 1, 2, 3, 16, 17
NONE, RMS = (0, 0, 0.0, 0, 0), (1, 0, 1e-6, 0x9000, 0)
STRIDES = (4096, 512, 64)
ROTATION = dict(pairs=32, pairing=0, axes=1, pos_type=I64, section=(32, 0, 0, 0), rows=10, ld=(32, 32), tables=(0x8000, 0x8800), positions=0x7000,
                pos=(0, 8, 1))


@pytest.fixture(scope="module")
def lib():
    return fo.load_library()


def rotation(**kw):
    r = {**ROTATION, **kw}
    return struct.pack("8i3q3Q3q", r["pairs"], r["pairing"], r["axes"], r["pos_type"], *r["section"], r["rows"], *r["ld"], *r["tables"],
                       r["positions"], *r["pos"])


def heads(heads=8, x=0x1000, y=0x2000, x_at=STRIDES, y_at=STRIDES, norm=RMS):
    return struct.pack("q2Q6qiidQQ", heads, x, y, *x_at, *y_at, *norm)


def head_norm(lib, batch=2, tokens=8, dim=64, type=BF16, vec=BF16, count=1, t=None, t2=None, rot=None):
    return lib.fused_head_norm(struct.pack("2q4i", batch, tokens, dim, type, vec, count) + (t or heads()) + (t2 or heads())
                               + (rot or rotation()), None)


def test_head_norm_refusals(lib):
    assert lib.fused_head_norm(None, None) == -1
    assert head_norm(lib, batch=-1) == -2 and head_norm(lib, tokens=-1) == -2 and head_norm(lib, dim=-1) == -2
    assert head_norm(lib, dim=513) == -4 and head_norm(lib, count=0) == -4 and head_norm(lib, count=3) == -4
    assert head_norm(lib, type=4) == -4 and head_norm(lib, type=F32, vec=BF16) == -4 and head_norm(lib, type=F64, vec=F32) == -4
    assert head_norm(lib, tokens=1 << 31) == -4 and head_norm(lib, tokens=1 << 28, t=heads(heads=100)) == -4
    assert head_norm(lib, t=heads(heads=-1)) == -2 and head_norm(lib, t=heads(x=0)) == -1 and head_norm(lib, t=heads(y=0)) == -1
    assert head_norm(lib, t=heads(x_at=(1, -1, 1))) == -2 and head_norm(lib, t=heads(y_at=(1, 1, -1))) == -2
    assert head_norm(lib, t=heads(x=0x1001)) == -4 and head_norm(lib, t=heads(norm=(1, 0, 1e-6, 0x9001, 0))) == -4
    assert head_norm(lib, t=heads(norm=(3, 0, 1e-6, 0, 0))) == -4 and head_norm(lib, t=heads(norm=(1, 0, -1.0, 0, 0))) == -4
    assert head_norm(lib, t=heads(norm=(2, 0, math.nan, 0, 0))) == -4 and head_norm(lib, count=2, t2=heads(x=0)) == -1
    for bad, code in ((dict(pairs=-1), -2), (dict(pairs=33), -2), (dict(pairing=2), -4), (dict(axes=0), -4), (dict(axes=5), -4), (dict(pos_type=1), -4),
                      (dict(section=(31, 0, 0, 0)), -2), (dict(axes=2, section=(40, -8, 0, 0)), -2), (dict(rows=-1), -2), (dict(ld=(31, 32)), -2),
                      (dict(ld=(32, 31)), -2), (dict(tables=(0, 0x8000)), -1), (dict(positions=0), -1), (dict(positions=0x7004), -4),
                      (dict(tables=(0x8000, 0x8002)), -4), (dict(pos=(0, -1, 1)), -2)):
        assert head_norm(lib, rot=rotation(**bad)) == code, bad
    assert head_norm(lib, batch=0) == 0 and head_norm(lib, dim=0, rot=rotation(pairs=0)) == 0 and head_norm(lib, t=heads(heads=0, x=0, y=0)) == 0


def head_grad(lib, t=None, ws=0x10000, ws_bytes=1 << 30, **kw):
    one = dict(heads=8, dy=0x1000, x=0x2000, dx=0x3000, norm=RMS, dw=0x4000, db=0)
    one.update(t or {})
    body = struct.pack("q3Q9qiidQQ2Q", one["heads"], one["dy"], one["x"], one["dx"], *STRIDES, *STRIDES, *STRIDES, *one["norm"], one["dw"], one["db"])
    top = dict(batch=2, tokens=8, dim=64, type=BF16, vec=BF16, count=1)
    top.update(kw)
    return lib.fused_head_norm_grad(struct.pack("2q4i", *top.values()) + body + body + rotation(), ws, ws_bytes, None)


def test_head_norm_grad_refusals(lib):
    assert lib.fused_head_norm_grad(None, None, 0, None) == -1
    assert head_grad(lib, dict(dy=0)) == -1 and head_grad(lib, dict(x=0)) == -1 and head_grad(lib, dict(dx=0)) == -1
    assert head_grad(lib, dict(norm=NONE)) == -1                 # the gradient of no weight
    assert head_grad(lib, dict(dw=0x4002)) == -4 and head_grad(lib, dict(dx=0x3001)) == -4
    assert head_grad(lib, dim=600) == -4 and head_grad(lib, batch=-1) == -2
    need = lib.fused_head_norm_grad_workspace_bytes
    assert need(64, BF16) > 16384 and need(-1, F32) == 0 and need(513, F32) == 0 and need(64, 9) == 0
    assert need(64, F64) - 16384 == 2 * (need(64, F32) - 16384)


def scan(lib, grad=False, **kw):
    v = dict(batch=2, tokens=8, channels=64, type=BF16, gate_type=BF16, decay=1, mix=1, x=0x1000, gate=0x2000, state=0, reset=0, lengths=0, at=(512, 64),
             gate_at=(512, 64), reset_at=(8, 1), lengths_type=I64, h=0x3000, last=0x4000, dh=0x5000, dlast=0, dx=0x6000, dgate=0x6800, dstate=0,
             ws=0x10000, ws_bytes=1 << 30)
    v.update(kw)
    head = struct.pack("3q4i", *(v[k] for k in ("batch", "tokens", "channels", "type", "gate_type", "decay", "mix")))
    if not grad:
        return lib.fused_scan(head + struct.pack("5Q6qii2Q2q", v["x"], v["gate"], v["state"], v["reset"], v["lengths"], *v["at"], *v["gate_at"],
                                                 *v["reset_at"], v["lengths_type"], 0, v["h"], v["last"], *v["at"]), v["ws"], v["ws_bytes"], None)
    return lib.fused_scan_grad(head + struct.pack("8Q10qii3Q4q", v["dh"], v["dlast"], v["x"], v["gate"], v["h"], v["state"], v["reset"], v["lengths"],
                                                  *v["at"], *v["at"], *v["gate_at"], *v["at"], *v["reset_at"], v["lengths_type"], 0, v["dx"], v["dgate"],
                                                  v["dstate"], *v["at"], *v["gate_at"]), v["ws"], v["ws_bytes"], None)


def test_scan_refusals(lib):
    assert lib.fused_scan(None, None, 0, None) == -1 and lib.fused_scan_grad(None, None, 0, None) == -1
    assert lib.fused_scan_workspace_bytes(1 << 30) > 16384 and lib.fused_scan_workspace_bytes(1) == 0
    for grad in (False, True):
        one = lambda **kw: scan(lib, grad, **kw)  # noqa: E731
        assert one(batch=-1) == -2 and one(tokens=-1) == -2 and one(channels=-1) == -2
        assert one(gate_type=F16) == -4 and one(type=F32) == -4 and one(type=F64, gate_type=F32) == -4 and one(type=7, gate_type=7) == -4
        assert one(decay=3) == -4 and one(decay=-1) == -4 and one(mix=3) == -4 and one(lengths=0x7000, lengths_type=2) == -4
        assert one(lengths=0x7004) == -4 and one(at=(-1, 64)) == -2 and one(gate_at=(512, -1)) == -2 and one(reset_at=(-8, 1)) == -2
        assert one(x=0) == -1 and one(gate=0) == -1 and one(h=0) == -1 and one(x=0x1001) == -4 and one(gate=0x2001) == -4
        assert one(state=0x7002) == -4 and one(batch=1 << 30, channels=1 << 20) == -4
        assert one(tokens=(1 << 30) + 1) == -4 and one(channels=(1 << 28) + 1) == -4
        for bad in (dict(ws=0), dict(ws=0x10008), dict(ws_bytes=16384)):
            assert one(tokens=9000, **bad) == -5
        assert one(batch=0) == 0 and one(channels=0) == 0 and one(tokens=0, last=0) == 0
    assert scan(lib, True, dx=0) == -1 and scan(lib, True, dgate=0) == -1 and scan(lib, True, dgate=0x6801) == -4 and scan(lib, True, dstate=0x6802) == -4
    assert scan(lib, last=0x4002) == -4


def distill(lib, what="fused_distill", **kw):
    v = dict(rows=4, vocab=1000, top=8, type=BF16, values_type=BF16, ids_type=I64, temperature=1.0, logits=0x1000, ids=0x2000, values=0x3000, tail=0, dloss=0,
             ld=(1000, 8, 8), loss=0x4000, stats=0x5000, dz=0x6000, ld_dz=1000)
    v.update(kw)
    return getattr(lib, what)(struct.pack("3q4id5Q3q3Qq", v["rows"], v["vocab"], v["top"], v["type"], v["values_type"], v["ids_type"], 0, v["temperature"],
                                          v["logits"], v["ids"], v["values"], v["tail"], v["dloss"], *v["ld"], v["loss"], v["stats"], v["dz"], v["ld_dz"]), None)


def test_distill_refusals(lib):
    for what in ("fused_distill", "fused_distill_grad", "fused_distill_step"):
        assert getattr(lib, what)(None, None) == -1
        one = lambda **kw: distill(lib, what, **kw)  # noqa: E731
        assert one(rows=-1) == -2 and one(vocab=-1) == -2 and one(top=-1) == -2 and one(top=1025, ld=(1000, 2000, 2000)) == -4
        assert one(type=4) == -4 and one(ids_type=F32) == -4 and one(values_type=F16) == -4 and one(type=F64, values_type=F32) == -4
        for t in (0.0, -1.0, math.nan, math.inf):
            assert one(temperature=t) == -4
        assert one(ld=(999, 8, 8)) == -2 and one(ld=(1000, 7, 8)) == -2 and one(ld=(1000, 8, 7)) == -2
        assert one(logits=0) == -1 and one(ids=0) == -1 and one(values=0) == -1
        assert one(logits=0x1001) == -4 and one(ids=0x2004) == -4 and one(values=0x3001) == -4 and one(tail=0x7002) == -4
        assert one(rows=0) == 0 and one(vocab=(1 << 20) + 1, ld=(1 << 21, 8, 8), ld_dz=1 << 21) == -4
        if what != "fused_distill":
            assert one(dz=0) == -1 and one(dz=0x6001) == -4 and one(ld_dz=999) == -2 and one(dloss=0x7002) == -4
        if what != "fused_distill_grad":
            assert one(loss=0x4002) == -4
    assert distill(lib, loss=0, stats=0) == -1 and distill(lib, "fused_distill_grad", stats=0) == -1 and distill(lib, "fused_distill_step", loss=0) == -1


def test_python_refusals():
    x = torch.zeros(4, 8)
    for call in (lambda: fo.fused_head_norm(x[None]), lambda: fo.fused_head_norm_grad(x[None]), lambda: fo.fused_scan(x, x),
                 lambda: fo.fused_scan_grad(x, x, x, x), lambda: fo.fused_distill(x, x.long(), x), lambda: fo.fused_distill_grad(None, x, x.long(), x, x),
                 lambda: fo.fused_distill_step(None, x, x.long(), x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    for call in (lambda: fo.fused_head_norm(None), lambda: fo.fused_head_norm_grad(), lambda: fo.fused_scan(None, x), lambda: fo.fused_scan(7, x),
                 lambda: fo.fused_scan_grad(None, x, x, x), lambda: fo.fused_distill(None, None, None)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_python_refusals_on_the_device():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    q, i64, bf = z(2, 5, 4, 16), torch.int64, torch.bfloat16
    cos, pos = z(9, 8), z(2, 5, dtype=i64)
    ok = (cos, cos, pos, "halves", None)
    fo.fused_head_norm(q, rotate=ok)
    bad = [dict(q=z(5, 16)), dict(q=z(1, 2, 5, 4, 16)), dict(q=z(2, 5, 4, 513)), dict(q=q.transpose(2, 3)), dict(q=q.int()), dict(k=z(2, 4, 4, 16)),
           dict(k=z(2, 5, 4, 8)), dict(k=z(2, 5, 4, 16, dtype=bf)), dict(k=z(5, 4, 16)), dict(k_norm=("rms", None, None, 1e-6)), dict(out_k=q),
           dict(q_norm=("norm", None, None, 1e-6)), dict(q_norm=("rms", z(8), None, 1e-6)), dict(q_norm=("rms", z(32)[::2], None, 1e-6)),
           dict(q_norm=("rms", z(16, dtype=bf), None, 1e-6)), dict(q_norm=("rms", None)), dict(out_q=z(2, 5, 4, 15)), dict(out_q=z(2, 5, 1, 16).expand(2, 5, 4, 16)),
           dict(out_q=z(2, 5, 4, 16, dtype=bf)), dict(rotate=(cos, cos, pos)), dict(rotate=(cos, z(9, 7), pos, "halves", None)),
           dict(rotate=(z(9, 9), z(9, 9), pos, "halves", None)), dict(rotate=(cos.double(), cos, pos, "halves", None)), dict(rotate=(cos, cos, pos.float(), "halves", None)),
           dict(rotate=(cos, cos, pos, "thirds", None)), dict(rotate=(cos, cos, pos, "halves", (4, 5))), dict(rotate=(cos, cos, pos, "halves", (4, 2, 2))),
           dict(rotate=(cos, cos, z(2, 2, 5, dtype=i64), "halves", (9, -1))), dict(rotate=(cos, cos, z(2, 2, 5, dtype=i64), "halves", [4, 4])),
           dict(rotate=(cos, cos, pos[:, :4], "halves", None)), dict(rotate=(cos, cos, pos[:1], "halves", None)), dict(rotate=(cos, cos, pos.cpu(), "halves", None)),
           dict(rotate=(z(8, 9).t(), cos, pos, "halves", None)), dict(q_norm=("rms", None, None, "small"))]
    for kw in bad:
        with pytest.raises((ValueError, TypeError)):
            fo.fused_head_norm(**{"q": q, **kw})
    for args, kw in (((q, None, None, None), dict(q_norm=("rms", None, None, 1e-6))), ((q, None, z(2, 5, 4, 8)), dict(q_norm=("rms", None, None, 1e-6))),
                     ((q, z(2, 5, 4, 8)), {}), ((None, q), dict(out_q=q))):
        with pytest.raises(ValueError):
            fo.fused_head_norm_grad(*args, **kw)
    x = z(2, 6, 8)
    fo.fused_scan(x, x)
    for args, kw in (((x, z(2, 6, 7)), {}), ((x, None), {}), ((z(8), z(8)), {}), ((x, x.to(bf)), {}), ((x.to(bf), z(2, 6, 8, dtype=torch.float16)), {}),
                     ((x, x, "relu"), {}), ((x, x, "exp", "all"), {}), ((x, x), dict(state=z(2, 7))), ((x, x), dict(state=z(2, 8, dtype=bf))),
                     ((x, x), dict(state=z(8, 2).t())), ((x, x), dict(reset=z(2, 6))), ((x, x), dict(reset=z(2, 5, dtype=torch.bool))),
                     ((x, x), dict(lengths=z(2))), ((x, x), dict(lengths=z(3, dtype=i64))), ((x, x), dict(lengths=torch.zeros(2, dtype=i64))),
                     ((z(2, 8, 6).transpose(1, 2), x), {}), ((x, x), dict(out=z(1, 6, 8).expand(2, 6, 8))), ((x, x), dict(out=z(2, 6, 9))),
                     ((x, x), dict(out_state=z(2, 8, dtype=torch.float64))), ((x.int(), x.int()), {})):
        with pytest.raises(ValueError):
            fo.fused_scan(*args, **kw)
    for args in ((None, x, x, x), (x, None, x, x), (x, x, x, None), (x, x, z(2, 6, 7), x), (z(2, 5, 8), x, x, x)):
        with pytest.raises(ValueError):
            fo.fused_scan_grad(*args)
    logits, ids, values = z(3, 50), z(3, 4, dtype=i64), z(3, 4)
    loss, stats = fo.fused_distill(logits, ids, values, stats=True)
    for args, kw in (((z(3), ids, values), {}), ((logits, ids.float(), values), {}), ((logits, ids[:2], values), {}), ((logits, ids, values[:, :3]), {}),
                     ((logits, ids, values.to(bf)), {}), ((logits.to(bf), ids, values.half()), {}), ((logits, ids, values), dict(tail=z(4))),
                     ((logits, ids, values), dict(tail=z(3, dtype=torch.float64))), ((z(50, 3).t(), ids, values), {}), ((z(1, 50).expand(3, 50), ids, values), {}),
                     ((logits, ids.cpu(), values), {}), ((logits.int(), ids, values), {})):
        with pytest.raises(ValueError):
            fo.fused_distill(*args, **kw)
    for kw in (dict(temperature=0.0), dict(temperature=float("nan"))):
        with pytest.raises(fo.FusedOpsError):
            fo.fused_distill(logits, ids, values, **kw)
    with pytest.raises(fo.FusedOpsError):
        fo.fused_distill(z(1, 1100), z(1, 1025, dtype=i64), z(1, 1025))
    for args in ((z(2), logits, ids, values, stats), (None, logits, ids, values, None), (None, logits, ids, values, stats[:2]),
                 (z(3, dtype=i64), logits, ids, values, stats)):
        with pytest.raises(ValueError):
            fo.fused_distill_grad(*args)
    with pytest.raises(ValueError):
        fo.fused_distill_step(None, logits, ids, values, out=z(3, 51))
    for shape, call in (((2, 6, 8), lambda t: fo.fused_scan(t, x)), ((2, 6, 8), lambda t: fo.fused_head_norm(t)),
                        ((6, 8), lambda t: fo.fused_distill(t, z(6, 1, dtype=i64), z(6, 1)))):
        with pytest.raises(ValueError, match="requires a gradient"):
            call(z(*shape).requires_grad_())
        shrunk = z(*shape)
        shrunk.untyped_storage().resize_(16)
        with pytest.raises(ValueError, match="storage"):
            call(shrunk)
