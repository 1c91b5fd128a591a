"""The training-step operators beside autograd: they record no graph, say so instead of losing a gradient, tell autograd
what they write, and work inside an autograd.Function."""
import pytest
import torch

import paper_1801_00829_b200 as fo

pytestmark = pytest.mark.gpu

EPS = 1e-6


def z(*s):
    return torch.rand(*s, device="cuda") + 0.1


@pytest.mark.parametrize("name", ["x", "f", "post", "post bias", "gate", "row gate", "col gate", "col_scale", "pre", "out_h", "out_y"])
def test_a_tensor_that_requires_a_gradient_is_refused(name):
    t = {k: z(4, 8) for k in ("x", "f", "gate", "out_h", "out_y")}
    t.update({k: z(8) for k in ("post", "post bias", "col gate", "col_scale", "pre")}, **{"row gate": z(4)})
    t[name].requires_grad_()
    access = name.split()[0] if name in ("row gate", "col gate") else "cell"
    gate = (access, t["gate" if access == "cell" else name], "silu")
    how = dict(post=("layer", t["post"], t["post bias"], EPS), gate=gate, col_scale=t["col_scale"], pre=("rms", t["pre"], None, EPS))
    with pytest.raises(ValueError, match="requires a gradient"):
        fo.fused_block_norm(t["x"], t["f"], out_h=t["out_h"], out_y=t["out_y"], **how)
    with torch.no_grad():
        h, y, stats = fo.fused_block_norm(t["x"], t["f"], out_h=t["out_h"], out_y=t["out_y"], stats=True, **how)
        fo.fused_block_norm_grad(h, y, h, t["f"], stats, **how)
    with torch.inference_mode():
        fo.fused_block_norm(t["x"], t["f"], **how)
    if name not in ("x", "out_h", "out_y"):
        with pytest.raises(ValueError, match="requires a gradient"):
            fo.fused_block_norm_grad(h.detach(), y.detach(), h.detach(), t["f"], stats, **how)


class BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, gate, post, pre):
        how = dict(post=("rms", post, None, EPS), gate=("cell", gate, "sigmoid"), scale=0.5, pre=("rms", pre, None, EPS))
        h, y, stats = fo.fused_block_norm(x, f, stats=True, **how)
        ctx.save_for_backward(h, f, gate, post, pre, stats)
        return h, y

    @staticmethod
    def backward(ctx, dh, dy):
        h, f, gate, post, pre, stats = ctx.saved_tensors
        how = dict(post=("rms", post, None, EPS), gate=("cell", gate, "sigmoid"), scale=0.5, pre=("rms", pre, None, EPS))
        got = fo.fused_block_norm_grad(dh.contiguous(), dy.contiguous(), h, f, stats, **how)
        return got["x"], got["f"], got["gate"], got["post_w"], got["pre_w"]


def test_inside_an_autograd_function():
    leaves = [z(6, 40), z(6, 40), z(6, 40), z(40), z(40)]
    for t in leaves:
        t.requires_grad_()
    h, y = BlockNorm.apply(*leaves)
    (h.square().sum() + y.sin().sum()).backward()
    got = [t.grad.clone() for t in leaves]
    wide = [t.detach().double().requires_grad_() for t in leaves]
    x, f, gate, post, pre = wide
    n = lambda t, w: t * torch.rsqrt(t.square().mean(1, keepdim=True) + EPS) * w  # noqa: E731
    h = x + 0.5 * torch.sigmoid(gate) * n(f, post)
    (h.square().sum() + n(h, pre).sin().sum()).backward()
    for a, t in zip(got, wide):
        assert (a.double() - t.grad).norm() <= 1e-5 * t.grad.norm()


def test_autograd_learns_what_was_written():
    """A tensor that autograd saved and a call then overwrites makes backward raise, as with any in-place operation."""
    def after(write):
        w = z(4, 8).requires_grad_()
        saved = z(4, 8)
        loss = (w * saved).sum()
        write(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()

    f, m, v = z(4, 8), z(4, 8), z(4, 8)
    after(lambda t: fo.fused_block_norm(t, f, out_h=t))
    after(lambda t: fo.fused_block_norm(f, pre=("rms", None, None, EPS), out_y=t))
    after(lambda t: fo.fused_grad_clip([t], 0.5))
    after(lambda t: fo.fused_grad_clip(fo.tensor_list([f], [t]), 0.5))
    after(lambda t: fo.fused_adamw(fo.adam_list([t], [f], [m], [v]), lr=0.1))
    after(lambda t: fo.fused_adamw(fo.adam_list([f], [f], [t], [v]), lr=0.1))
    after(lambda t: fo.fused_adamw(fo.adam_list([f], [f], [m], [v], outs=([z(4, 8)], [z(4, 8)], [t])), lr=0.1))
    low = z(4, 8).to(torch.bfloat16)
    version = low._version
    fo.fused_adamw(fo.adam_list([f], [f], [m], [v], weights=[low]), lr=0.1)
    assert low._version == version + 1


def test_what_is_only_read_keeps_its_version():
    x, f, w, g = z(4, 8), z(4, 8), z(8), z(100)
    kept = fo.tensor_list([g], [z(100)])
    before = [t._version for t in (x, f, w, g)]
    fo.fused_block_norm(x, f, post=("rms", w, None, EPS))
    fo.fused_grad_norm([g], 1.0)
    fo.fused_grad_norm(kept, 1.0)
    fo.fused_grad_clip(kept, 1.0)
    fo.adam_list([g], [g], [g], [g])
    assert [t._version for t in (x, f, w, g)] == before


def test_parameters_are_updated_while_gradients_are_recorded():
    """As an optimiser does: the update is no part of the graph."""
    p = torch.nn.Parameter(z(300))
    (p * 2.0).sum().backward()
    m, v = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    before = p.detach().clone()
    result = fo.fused_grad_clip([p.grad], 1e9)
    fo.fused_adamw(fo.adam_list([p], [p.grad], [m], [v]), lr=0.1, factor=result[1:])
    assert torch.allclose(p.detach(), before - 0.1, rtol=0, atol=1e-5)


def test_tensors_of_inference_mode():
    with torch.inference_mode():
        x, f = z(4, 8), z(4, 8)
    h, _, _ = fo.fused_block_norm(x, f, out_h=x)
    assert h is x and fo.fused_grad_clip([x], 1e9)[1].item() == 1.0
