"""Refusals of the training-step operators: found on the host, before anything is launched (no GPU needed)."""
import math
import struct

import pytest
import torch

import paper_1801_00829_b200 as fo

# fo_block_norm and fo_block_norm_grad, field by field
BLOCK_NORM = struct.Struct("qq6i4Q3qd" + "iidQQ" * 2 + "3Q2q")
BLOCK_NORM_GRAD = struct.Struct("qq6i7Q5qd" + "iidQQ" * 2 + "3Q3q5Q")
NONE = (0, 0, 0.0, 0, 0)
RMS = (1, 0, 1e-6, 0x9000, 0)
F64, F32, BF16, F16 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    return fo.load_library()


def norm(lib, rows=4, cols=64, types=(BF16, BF16, BF16), access=0, act=0, x=0x1000, f=0x2000, gate=0, col_scale=0,
         ld=(64, 64, 64), post=RMS, pre=RMS, h=0x3000, y=0x4000, stats=0, ld_out=(64, 64)):
    return lib.fused_block_norm(BLOCK_NORM.pack(rows, cols, *types, access, act, 0, x, f, gate, col_scale, *ld, 1.0, *post,
                                                   *pre, h, y, stats, *ld_out), None)


def test_block_norm_refusals(lib):
    assert lib.fused_block_norm(None, None) == -1
    assert norm(lib, rows=-1) == -2 and norm(lib, cols=-1) == -2
    assert norm(lib, cols=32769, ld=(1 << 16,) * 3, ld_out=(1 << 16,) * 2) == -4
    assert norm(lib, rows=1 << 31) == -4
    assert norm(lib, ld=(63, 64, 64)) == -2 and norm(lib, ld=(64, 63, 64)) == -2
    assert norm(lib, ld_out=(63, 64)) == -2 and norm(lib, ld_out=(64, 63)) == -2
    assert norm(lib, gate=0x5000, ld=(64, 64, 63)) == -2
    assert norm(lib, gate=0x5000, access=1, ld=(64, 64, 0)) == -2
    assert norm(lib, gate=0x5000, access=3) == -4 and norm(lib, gate=0x5000, act=4) == -4
    assert norm(lib, x=0, f=0, post=NONE) == -1
    assert norm(lib, f=0) == -1                                  # a post norm without a block
    assert norm(lib, f=0, post=NONE, gate=0x5000) == -1
    assert norm(lib, h=0, y=0) == -1                             # nothing wanted
    assert norm(lib, pre=NONE) == -1                             # y without its norm
    assert norm(lib, post=(3, 0, 1e-6, 0, 0)) == -4
    assert norm(lib, post=(1, 0, -1e-6, 0, 0)) == -4 and norm(lib, pre=(1, 0, math.nan, 0, 0)) == -4
    for types in ((BF16, F16, F16), (BF16, F32, F32), (F64, F32, F32), (F32, F64, F64), (4, 4, 4), (BF16, BF16, F16), (F32, F32, BF16),
                  (F64, F64, F32)):
        assert norm(lib, types=types) == -4
    assert norm(lib, rows=0, x=0, f=0) == 0 and norm(lib, cols=0) == 0      # nothing to do


def grad(lib, rows=4, cols=64, types=(BF16, BF16, BF16), access=0, act=0, dh=0x1000, dy=0x1100, h=0x1200, f=0x1300, gate=0,
         col_scale=0, stats=0x1400, ld=(64,) * 5, post=RMS, pre=RMS, dx=0x1500, df=0x1600, dgate=0, ld_out=(64,) * 3,
         sums=(0, 0, 0, 0, 0), ws=0x10000, ws_bytes=1 << 30):
    return lib.fused_block_norm_grad(BLOCK_NORM_GRAD.pack(rows, cols, *types, access, act, 0, dh, dy, h, f, gate, col_scale,
                                                             stats, *ld, 1.0, *post, *pre, dx, df, dgate, *ld_out, *sums),
                                     ws, ws_bytes, None)


def test_block_norm_grad_refusals(lib):
    assert lib.fused_block_norm_grad(None, None, 0, None) == -1
    assert grad(lib, rows=-1) == -2 and grad(lib, cols=32769) == -4
    assert grad(lib, dh=0, dy=0) == -1
    assert grad(lib, h=0) == -1 and grad(lib, stats=0) == -1
    assert grad(lib, pre=NONE) == -1                             # dy without its norm
    assert grad(lib, pre=NONE, dy=0, sums=(0, 0, 0, 0x7000, 0)) == -1
    assert grad(lib, f=0, post=NONE, df=0x1600) == -1 and grad(lib, f=0, df=0) == -1
    assert grad(lib, dgate=0x1700) == -1                         # a gradient of no gate
    assert grad(lib, post=NONE, sums=(0, 0x7000, 0, 0, 0)) == -1
    for k in range(4):
        assert grad(lib, ld=tuple(63 if i == k else 64 for i in range(5))) == -2
    assert grad(lib, ld_out=(63, 64, 64)) == -2 and grad(lib, ld_out=(64, 63, 64)) == -2
    assert grad(lib, gate=0x1800, dgate=0x1700, ld_out=(64, 64, 63)) == -2
    assert grad(lib, types=(BF16, F16, F16)) == -4
    assert grad(lib, ws=0) == -5 and grad(lib, ws=0x10008) == -5 and grad(lib, ws_bytes=16384) == -5
    need = lib.fused_block_norm_grad_workspace_bytes
    assert need(4, 64, BF16) >= 16384 + 6 * 4 * 64 * 4
    assert need(4, 64, F64) - 16384 == 2 * (need(4, 64, BF16) - 16384)
    assert need(-1, 64, BF16) == 0 and need(4, 64, 9) == 0 and need(4, 40000, BF16) == 0


def test_many_tensor_refusals(lib):
    one = struct.pack("QQq", 0x1000, 0x2000, 10)
    ws, big = 0x10000, 1 << 20
    norm_ = lambda t=one, n=1, it=F32, kind=0, mx=1.0, eps=0.0, res=0x3000, rt=F32, w=ws, wb=big: lib.fused_grad_norm(  # noqa: E731
        t, n, it, kind, mx, eps, res, rt, w, wb, None)
    assert norm_(t=None) == -1 and norm_(n=-1) == -2 and norm_(it=7) == -4 and norm_(kind=2) == -4 and norm_(rt=BF16) == -4
    assert norm_(mx=-1.0) == -2 and norm_(mx=math.nan) == -2 and norm_(eps=-1.0) == -2 and norm_(res=0) == -1
    assert norm_(w=0) == -5 and norm_(wb=64) == -5
    assert norm_(t=struct.pack("QQq", 0, 0, 10)) == -1 and norm_(t=struct.pack("QQq", 0x1000, 0, -1)) == -2
    clip = lambda t=one, it=F32, ot=F32: lib.fused_grad_clip(t, 1, it, ot, 0, 1.0, 0.0, 0x3000, F32, ws, big, None)  # noqa: E731
    assert clip(ot=BF16) == -4 and clip(it=BF16, ot=F16) == -4 and clip(it=F64, ot=F32) == -4 and clip(ot=9) == -4
    assert clip(t=struct.pack("QQq", 0x1000, 0, 10)) == -1
    adam = struct.pack("8Qqd", *([0x1000] * 8), 10, 0.0)
    step = lambda t=adam, n=1, g=F32, w=BF16, b1=0.9, b2=0.99, eps=1e-8, s=1, f=0, ft=F32: lib.fused_adamw(  # noqa: E731
        t, n, g, w, 1e-3, b1, b2, eps, s, f, ft, None)
    assert step(t=None) == -1 and step(n=-1) == -2 and step(g=9) == -4 and step(w=F32) == -4 and step(g=F64) == -4
    assert step(b1=1.0) == -2 and step(b2=-0.1) == -2 and step(eps=-1.0) == -2 and step(s=0) == -2 and step(f=0x10, ft=BF16) == -4
    assert step(t=struct.pack("8Qqd", 0x1000, 0, *([0x1000] * 6), 10, 0.0)) == -1


def test_python_refusals():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        fo.fused_block_norm(x, pre=("rms", None, None, 1e-6))
    with pytest.raises(ValueError, match="CUDA"):
        fo.fused_grad_norm([x], 1.0)
    with pytest.raises(ValueError, match="x or f"):
        fo.fused_block_norm()
    with pytest.raises(ValueError, match="dh or dy"):
        fo.fused_block_norm_grad()


@pytest.mark.gpu
def test_python_refusals_on_the_device():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    x = z(4, 8)
    bad = [dict(x=x, f=z(4, 9)), dict(x=x, f=z(5, 8)), dict(x=x, f=z(4, 8, dtype=torch.float64)),
           dict(x=z(4, 8, dtype=torch.bfloat16), f=x), dict(x=z(8, 4).t(), f=x), dict(x=x, post=("rms", None, None, 1e-6)),
           dict(x=x, f=x, pre=("norm", None, None, 1e-6)), dict(x=x, pre=("rms", z(7), None, 1e-6)),
           dict(x=x, pre=("rms", z(16)[::2], None, 1e-6)), dict(x=x, f=x, gate=("cell", z(4, 7), "silu")),
           dict(x=x, f=x, gate=("row", z(8), "silu")), dict(x=x, f=x, gate=("row", z(4), "relu")),
           dict(x=x, f=x, gate=("all", z(4), "silu")), dict(x=x, f=x, col_scale=z(8, dtype=torch.bfloat16)),
           dict(x=x, f=x, out_y=z(4, 8)), dict(x=z(8), f=None), dict(x=z(1, 8).expand(4, 8), f=x)]
    for kw in bad:
        with pytest.raises(ValueError):
            fo.fused_block_norm(**kw)
    with pytest.raises(ValueError):
        fo.fused_block_norm_grad(x, x, None, None, pre=("rms", None, None, 1e-6))
    with pytest.raises(ValueError):
        fo.fused_block_norm_grad(x, x, x, None, z(4, 5), pre=("rms", None, None, 1e-6))
    with pytest.raises(ValueError):
        fo.tensor_list([x, z(3, dtype=torch.float16)])
    with pytest.raises(ValueError):
        fo.tensor_list([x], [z(31)])
    with pytest.raises(ValueError):
        fo.tensor_list([x.t()])
    with pytest.raises(ValueError):
        fo.tensor_list([x], [z(32, dtype=torch.bfloat16)])
    with pytest.raises(ValueError):
        fo.adam_list([x], [x], [x], [x], decay=[0.0, 0.1])
    with pytest.raises(ValueError):
        fo.adam_list([x], [z(4, 8, dtype=torch.float64)], [x], [x])
