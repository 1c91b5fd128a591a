"""The example that runs the training-step operators together: it learns, its backward pass is the gradient of
its forward pass, and a token gets the same answer alone and in a batch."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns(example):
    losses, one, row = example.train(steps=60)
    assert all(v == v for v in losses) and losses[-1] < 0.5 * losses[0]
    # the products may add up in another order for one row: a few roundings to bfloat16 of values around 1
    assert (one.float() - row.float()).abs().max().item() <= 0.1


def test_backward_is_the_gradient_of_forward(example):
    """Against automatic differentiation of the same network in float32, operator by operator; bfloat16
    activations and weights leave a few parts in a hundred."""
    torch.manual_seed(1)
    model = example.Model(128, 192, 2)
    x = torch.randn(96, 128, device="cuda")
    target = torch.randn(96, 128, device="cuda")
    kept = []
    error = model.forward(x, kept).float() - target
    model.backward((error * (2.0 / error.numel())).to(torch.bfloat16), kept)

    leaves = {name: low.float().requires_grad_() for name, low in zip(model.names, model.low)}

    def norm(t, w):
        return t * torch.rsqrt(t.square().mean(1, keepdim=True) + example.EPS) * w

    h, y = x, norm(x, leaves["first", 0])
    for k in range(2):
        f = torch.nn.functional.silu(y @ leaves["w1", k]) @ leaves["w2", k]
        h = h + example.SCALE * leaves["cs", k] * torch.sigmoid(y @ leaves["wg", k]) * norm(f, leaves["post", k])
        y = norm(h, leaves["pre", k])
    (y - target).square().mean().backward()
    for (name, got) in zip(model.names, model.grad):
        want = leaves[name].grad
        assert (got - want).norm() <= 0.05 * want.norm(), name
