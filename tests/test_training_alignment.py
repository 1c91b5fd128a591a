"""Addresses that are not those of an element are refused on the host, before anything is launched (no GPU needed): the
kernels read and write whole elements."""
import struct

import pytest

import paper_1801_00829_b200 as fo
from test_training_abi import BF16, F16, F32, F64, grad, norm

TYPES = [(F64, F64, F64), (F32, F32, F32), (BF16, BF16, BF16), (F16, F16, F16), (F32, BF16, BF16), (F32, F16, F32)]
SIZE = {F64: 8, F32: 4, BF16: 2, F16: 2}


@pytest.fixture(scope="module")
def lib():
    return fo.load_library()


@pytest.mark.parametrize("types", TYPES)
def test_block_norm(lib, types):
    stream, block, vec = types
    full = dict(gate=0x5000, col_scale=0x6000, stats=0x7000, post=(1, 0, 1e-6, 0x9000, 0xa000), pre=(2, 0, 1e-6, 0xb000, 0xc000))
    sums = F64 if block == F64 else F32
    for name, address, type_ in (("x", 0x1000, stream), ("f", 0x2000, block), ("gate", 0x5000, block), ("col_scale", 0x6000, vec),
                                 ("h", 0x3000, stream), ("y", 0x4000, block), ("stats", 0x7000, sums)):
        assert norm(lib, types=types, **{**full, name: address + SIZE[type_] // 2}) == -4, name
    for part in ("post", "pre"):
        for at in (3, 4):
            spec = list(full[part])
            spec[at] += SIZE[vec] // 2
            assert norm(lib, types=types, **{**full, part: tuple(spec)}) == -4, (part, at)


@pytest.mark.parametrize("types", TYPES)
def test_block_norm_grad(lib, types):
    stream, block, vec = types
    sums = F64 if block == F64 else F32
    outs = (0x20000, 0x21000, 0x22000, 0x23000, 0x24000)
    full = dict(gate=0x5000, dgate=0x1700, col_scale=0x6000, sums=outs, post=(1, 0, 1e-6, 0x9000, 0xa000), pre=(2, 0, 1e-6, 0xb000, 0xc000))
    for name, address, type_ in (("dh", 0x1000, stream), ("dy", 0x1100, block), ("h", 0x1200, stream), ("f", 0x1300, block),
                                 ("gate", 0x5000, block), ("col_scale", 0x6000, vec), ("stats", 0x1400, sums), ("dx", 0x1500, stream),
                                 ("df", 0x1600, block), ("dgate", 0x1700, block)):
        assert grad(lib, types=types, **{**full, name: address + SIZE[type_] // 2}) == -4, name
    assert grad(lib, types=types, access=1, **{**full, "dgate": 0x1700 + SIZE[sums] // 2}) == -4
    for k in range(5):
        assert grad(lib, types=types, **{**full, "sums": outs[:k] + (outs[k] + SIZE[sums] // 2,) + outs[k + 1:]}) == -4
    for part in ("post", "pre"):
        for at in (3, 4):
            spec = list(full[part])
            spec[at] += SIZE[vec] // 2
            assert grad(lib, types=types, **{**full, part: tuple(spec)}) == -4, (part, at)


@pytest.mark.parametrize("in_type,out_type", [(F64, F64), (F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)])
def test_lists(lib, in_type, out_type):
    good = struct.pack("QQq", 0x1000, 0x2000, 10)

    def call(more, clip=True, result=0x3000, result_type=F32):
        rest = (in_type, out_type) if clip else (in_type,)
        return (lib.fused_grad_clip if clip else lib.fused_grad_norm)(good + more, 2, *rest, 0, 1.0, 0.0, result, result_type, 0x10000,
                                                                      1 << 20, None)

    odd_in = struct.pack("QQq", 0x4000 + SIZE[in_type] // 2, 0x5000, 10)
    assert call(odd_in) == -4 and call(odd_in, clip=False) == -4
    assert call(struct.pack("QQq", 0x4000, 0x5000 + SIZE[out_type] // 2, 10)) == -4
    assert call(good, result=0x3002) == -4 and call(good, result=0x3004, result_type=F64) == -4


@pytest.mark.parametrize("grad_type,weight_type", [(F64, 0), (F32, BF16), (BF16, BF16), (F16, F16)])
def test_adamw(lib, grad_type, weight_type):
    wide = F64 if grad_type == F64 else F32
    sizes = [SIZE[wide], SIZE[grad_type]] + [SIZE[wide]] * 5 + ([2] if weight_type else [])
    for k, size in enumerate(sizes):
        at = [0x1000 * (i + 1) for i in range(8)]
        at[7] = at[7] if weight_type else 0
        at[k] += size // 2
        assert lib.fused_adamw(struct.pack("8Qqd", *at, 10, 0.0), 1, grad_type, weight_type, 1e-3, 0.9, 0.99, 1e-8, 1, 0, F32, None) == -4
    good = struct.pack("8Qqd", *[0x1000 * (i + 1) for i in range(7)], 0, 10, 0.0)
    assert lib.fused_adamw(good, 1, grad_type, weight_type, 1e-3, 0.9, 0.99, 1e-8, 1, 0x2002, F32, None) == -4
