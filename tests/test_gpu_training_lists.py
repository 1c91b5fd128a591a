"""Lists of tensors that are kept while their tensors change: every call works on what the tensors are at that time, and
refuses what does not fit.  Values as in test_gpu_training.py."""
import pytest
import torch

import paper_1801_00829_b200 as fo

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def grads(dtype=F32):
    return [torch.full((n,), v, dtype=dtype, device="cuda") for n, v in ((9000, 1.0), (5, 2.0), (0, 0.0), (300, 0.0))]


def norm_of(kept):
    return fo.fused_grad_norm(kept, 1.0, result_type=torch.float64)[0].item()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_storage_swapped_between_calls(dtype):
    g = grads(dtype)
    kept = fo.tensor_list(g)
    assert norm_of(kept) == pytest.approx(9020 ** 0.5, rel=1e-6)
    old = g[1]
    g[1].data = torch.full((5,), 4.0, dtype=dtype, device="cuda")
    assert old is kept.grads[1] and norm_of(kept) == pytest.approx(9080 ** 0.5, rel=1e-6)
    with torch.no_grad():
        g[0].set_(torch.full((9000,), 2.0, dtype=dtype, device="cuda"))
    assert norm_of(kept) == pytest.approx(36080 ** 0.5, rel=1e-6)
    result = fo.fused_grad_clip(kept, 1.0)
    scale = result[1].item()
    assert scale < 1.0 and g[0][17].item() == pytest.approx(2.0 * scale, rel=2.0 ** -8) and bool((g[0] == g[0][17]).all())


def test_outs_swapped_between_calls():
    g, outs = grads(), [torch.zeros(n, device="cuda") for n in (9000, 5, 0, 300)]
    kept = fo.tensor_list(g, outs)
    fo.fused_grad_clip(kept, 1e9)
    first = outs[0].detach()
    outs[0].data = torch.zeros(9000, device="cuda")
    g[0].fill_(3.0)
    fo.fused_grad_clip(kept, 1e9)
    assert bool((first == 1.0).all()) and bool((outs[0] == 3.0).all())


def test_a_tensor_that_no_longer_fits_is_refused():
    def swapped(value):
        g = grads()
        kept = fo.tensor_list(g, [torch.zeros_like(t) for t in g])
        g[0].data = value
        return kept

    for value in (torch.ones(8000, device="cuda"), torch.ones(9000, device="cuda").double(), torch.ones(9000),
                  torch.ones(18000, device="cuda")[::2]):
        with pytest.raises(ValueError):
            fo.fused_grad_clip(swapped(value), 1.0)
    g = grads()
    kept = fo.tensor_list(g)
    g[0].untyped_storage().resize_(0)
    for call in (fo.fused_grad_norm, fo.fused_grad_clip):
        with pytest.raises(ValueError, match="storage"):
            call(kept, 1.0)
    g[0].untyped_storage().resize_(9000 * 4)
    g[0].fill_(2.0)
    assert norm_of(kept) == pytest.approx(36020 ** 0.5, rel=1e-6)
    with pytest.raises(ValueError):
        fo.tensor_list([g[0], None])


@pytest.mark.parametrize("in_place", [True, False])
def test_adamw_with_storage_swapped_between_calls(in_place):
    sizes = (4099, 64, 1, 0)

    def fill(v):
        return [torch.full((n,), v, device="cuda") for n in sizes]

    p, g, m, v = fill(1.0), fill(0.5), fill(0.0), fill(0.0)
    outs = None if in_place else (fill(7.0), fill(7.0), fill(7.0))
    w = [t.to(BF16) for t in p]
    kept = fo.adam_list(p, g, m, v, outs=outs, weights=w)
    fo.fused_adamw(kept, lr=0.1, step=1)
    po = (outs or (p,))[0]
    assert all(torch.allclose(t, torch.full_like(t, 0.9), rtol=0, atol=1e-6) for t in po)
    behind = [t.detach() for t in po]
    for t in (*p, *m, *v):                                  # all of it moves; the old memory stays as it is
        t.data = torch.zeros_like(t)
    if outs:
        for t in outs[0]:
            t.data = torch.zeros_like(t)
    g[0].data = torch.full((sizes[0],), -2.0, device="cuda")
    fo.fused_adamw(kept, lr=0.1, step=1)
    assert all(torch.allclose(t, torch.full_like(t, 0.9), rtol=0, atol=1e-6) for t in behind)
    assert torch.allclose(po[0], torch.full_like(po[0], 0.1), rtol=0, atol=1e-6)
    assert torch.allclose(po[1], torch.full_like(po[1], -0.1), rtol=0, atol=1e-6)
    assert all(torch.equal(a, b.to(BF16)) for a, b in zip(w, po))
    m[1].data = torch.zeros(63, device="cuda")
    with pytest.raises(ValueError, match="m: sizes differ"):
        fo.fused_adamw(kept, lr=0.1, step=1)
    m[1].data = torch.zeros(64, device="cuda")
    w[0].untyped_storage().resize_(0)
    with pytest.raises(ValueError, match="weights: .*storage"):
        fo.fused_adamw(kept, lr=0.1, step=1)


def test_refused_lists():
    z = lambda n, dtype=F32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    with pytest.raises(ValueError):
        fo.adam_list([z(3)], [z(3)], [z(3)], [])
    with pytest.raises(ValueError):
        fo.adam_list([z(3)], [z(3)], [z(3)], [z(4)])
    with pytest.raises(ValueError):
        fo.adam_list([z(3)], [z(3)], [z(3)], [z(3)], weights=[z(3)])
    with pytest.raises(ValueError):
        fo.adam_list([z(3)], [z(3)], [z(3)], [z(3)], outs=([z(3)], [z(3)]))
    with pytest.raises(ValueError):
        fo.adam_list([z(3)], [z(3, torch.int32)], [z(3)], [z(3)])
    with pytest.raises(ValueError):
        fo.tensor_list([z(3), 1.0])
    with pytest.raises(ValueError):
        fo.tensor_list([z(3, torch.float64)], [z(3)])


@pytest.mark.parametrize("dtype", [torch.float64, F32, BF16, torch.float16])
@pytest.mark.parametrize("kind", ["l2", "max"])
@pytest.mark.parametrize("most", [0.75, 1e9])
def test_clipped_in_place(dtype, kind, most):
    """In place the values are those of the same call into other tensors, bit for bit, and with a factor of 1 the ones that
    were there; beside float32 outs, the same rounded once."""
    torch.manual_seed(7)
    sizes = (1, 0, 3, 7, 17, 8193, 100003)
    wide = torch.float64 if dtype == torch.float64 else F32
    for shift in (0, 1):
        flat = torch.randn(sum(sizes) + shift, device="cuda").to(dtype)[shift:]
        for g in (list(torch.split(flat, sizes)), [t.clone() for t in torch.split(flat, sizes)]):
            was = [t.clone() for t in g]
            same, more = [torch.zeros_like(t) for t in g], [torch.zeros(t.shape, dtype=wide, device="cuda") for t in g]
            a = fo.fused_grad_clip(fo.tensor_list(g, same), most, kind=kind, result_type=wide)
            b = fo.fused_grad_clip(fo.tensor_list(g, more), most, kind=kind, result_type=wide)
            c = fo.fused_grad_clip(g, most, kind=kind, result_type=wide)
            assert torch.equal(a, b) and torch.equal(a, c) and (c[1].item() == 1.0) == (most == 1e9)
            for now, other, wider, before in zip(g, same, more, was):
                assert torch.equal(now, other) and torch.equal(now, wider.to(dtype)) and torch.equal(wider, before.to(wide) * c[1])
                assert most < 1.0 or torch.equal(now, before)


@pytest.mark.parametrize("device", ["cuda", "cuda:0", 0, torch.device("cuda"), None])
def test_the_device_of_an_empty_list(device):
    for call in (fo.fused_grad_norm, fo.fused_grad_clip):
        result = call([], 1.0, device=device)
        assert result.device == torch.device("cuda", 0) and result.tolist() == [0.0, 1.0]


def test_a_device_without_kernels_is_refused():
    for call in (fo.fused_grad_norm, fo.fused_grad_clip):
        with pytest.raises(ValueError, match="CUDA"):
            call([], 1.0, device="cpu")


@pytest.mark.parametrize("name", ["x", "f", "post", "gate", "row gate", "col_scale", "pre", "out_h", "out_y", "dh", "dy", "h", "stats",
                                  "factor"])
def test_a_tensor_without_its_storage_is_refused(name):
    """What sharded trainers leave of a parameter between two uses: a tensor whose storage was resized to nothing."""
    z = lambda *s: torch.rand(*s, device="cuda") + 0.1  # noqa: E731
    t = {k: z(4, 8) for k in ("x", "f", "gate", "out_h", "out_y", "dh", "dy", "h")}
    t.update({k: z(8) for k in ("post", "col_scale", "pre")}, stats=z(4, 4), factor=z(1), **{"row gate": z(4)})
    gate = ("row", t["row gate"], "silu") if name == "row gate" else ("cell", t["gate"], "silu")
    how = dict(post=("rms", t["post"], None, 1e-6), gate=gate, col_scale=t["col_scale"], pre=("rms", t["pre"], None, 1e-6))
    adam = fo.adam_list(*[[z(5)] for _ in range(4)])
    calls = [lambda: fo.fused_block_norm(t["x"], t["f"], out_h=t["out_h"], out_y=t["out_y"], **how),
             lambda: fo.fused_block_norm_grad(t["dh"], t["dy"], t["h"], t["f"], t["stats"], **how),
             lambda: fo.fused_adamw(adam, lr=0.1, factor=t["factor"])]
    for call in calls:
        call()
    t[name].untyped_storage().resize_(0)
    refused = 0
    for call in calls:
        try:
            call()
        except ValueError as e:
            assert "storage" in str(e)
            refused += 1
    assert refused == (2 if name in ("f", "post", "gate", "row gate", "col_scale", "pre") else 1)
