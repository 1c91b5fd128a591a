"""Trains a few gated residual blocks with the training-step operators, then runs them for a single token.

    python examples/train_block.py [steps]

Every block is  x <- x + scale * col_scale * sigmoid(y Wg) * norm(silu(y W1) W2),  y = norm(x): the norm after the
block, its gate, the residual scale, the addition and the next block's norm are one fused_block_norm call
forward and one fused_block_norm_grad call backward.  The step's update takes the clipping factor of the global
gradient norm straight from the device.  The stream is in 32 bits, the blocks are in bfloat16, with 32-bit masters.
The task: map random tokens to the outputs of a random linear map.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1801_00829_b200 as fo  # noqa: E402

BLOCK, EPS, SCALE = torch.bfloat16, 1e-6, 0.5


def silu_grad(a):
    s = torch.sigmoid(a)
    return s * (1.0 + a * (1.0 - s))


class Model:
    """Weights as views into one bucket per kind (masters, moments, bfloat16 copies), as an optimiser keeps them."""

    def __init__(self, width, hidden, layers, device="cuda"):
        shapes = []
        for k in range(layers):
            shapes += [("w1", k, (width, hidden)), ("w2", k, (hidden, width)), ("wg", k, (width, width)),
                       ("post", k, (width,)), ("pre", k, (width,)), ("cs", k, (width,))]
        shapes.append(("first", 0, (width,)))
        self.width, self.layers = width, layers
        self.names = [(n, k) for n, k, _ in shapes]
        sizes = [int(torch.Size(s).numel()) for _, _, s in shapes]

        def bucket(dtype):
            parts = torch.zeros(sum(sizes), dtype=dtype, device=device).split(sizes)
            return [p.view(s) for p, (_, _, s) in zip(parts, shapes)]

        self.master, self.m, self.v, self.low = bucket(torch.float32), bucket(torch.float32), bucket(torch.float32), bucket(BLOCK)
        self.grad = bucket(torch.float32)
        for (name, _, shape), p in zip(shapes, self.master):
            if len(shape) == 2:
                p.normal_(0.0, shape[0] ** -0.5)
            else:
                p.fill_(0.5 if name == "cs" else 1.0)
        for low, p in zip(self.low, self.master):
            low.copy_(p)
        decay = [0.01 if len(shape) == 2 else 0.0 for _, _, shape in shapes]
        self.gradients = fo.tensor_list(self.grad)
        self.update = fo.adam_list(self.master, self.grad, self.m, self.v, decay=decay, weights=self.low)

    def weight(self, name, k):
        return self.low[self.names.index((name, k))]

    def how(self, k, gate):
        """The arguments that end block k and begin block k + 1."""
        return dict(post=("rms", self.weight("post", k), None, EPS), gate=("cell", gate, "sigmoid"), scale=SCALE,
                    col_scale=self.weight("cs", k), pre=("rms", self.weight("pre", k), None, EPS))

    def forward(self, x, keep=None):
        """The last norm's output; `keep`: a list that takes what the backward pass needs."""
        first = ("rms", self.weight("first", 0), None, EPS)
        _, y, stats = fo.fused_block_norm(x, pre=first, block_type=BLOCK, stats=keep is not None)
        if keep is not None:
            keep.append((x, stats, first))
        for k in range(self.layers):
            a = y @ self.weight("w1", k)
            s = torch.nn.functional.silu(a)
            f, gate = s @ self.weight("w2", k), y @ self.weight("wg", k)
            x, y_next, stats = fo.fused_block_norm(x, f, stats=keep is not None, **self.how(k, gate))
            if keep is not None:
                keep.append((y, a, s, f, gate, x, stats))
            y = y_next
        return y

    def backward(self, dy, kept):
        """Fills self.grad from the gradient of the last norm's output."""
        grad = {name: g for name, g in zip(self.names, self.grad)}
        dh = None
        for k in reversed(range(self.layers)):
            y, a, s, f, gate, h, stats = kept[k + 1]
            got = fo.fused_block_norm_grad(dh, dy, h, f, stats, **self.how(k, gate))
            for name, key in (("post", "post_w"), ("pre", "pre_w"), ("cs", "col_scale")):
                grad[name, k].copy_(got[key])
            df, dgate, dh = got["f"], got["gate"], got["x"]
            da = (df @ self.weight("w2", k).t()) * silu_grad(a)
            grad["w2", k].copy_(s.t() @ df)
            grad["w1", k].copy_(y.t() @ da)
            grad["wg", k].copy_(y.t() @ dgate)
            dy = da @ self.weight("w1", k).t() + dgate @ self.weight("wg", k).t()
        x, stats, first = kept[0]
        grad["first", 0].copy_(fo.fused_block_norm_grad(dh, dy, x, stats=stats, pre=first)["pre_w"])

    def step(self, x, target, number, lr=3e-3, max_norm=1.0):
        """One training step; the loss as a tensor on the device."""
        kept = []
        error = self.forward(x, kept).float() - target
        self.backward((error * (2.0 / error.numel())).to(BLOCK), kept)
        result = fo.fused_grad_norm(self.gradients, max_norm)
        fo.fused_adamw(self.update, lr=lr, step=number, factor=result[1:])
        return error.square().mean()


def train(steps=60, tokens=512, width=256, hidden=512, layers=3, seed=0):
    """Losses of the steps, and the trained model's answer to one token beside its row of the whole batch."""
    torch.manual_seed(seed)
    model = Model(width, hidden, layers)
    x = torch.randn(tokens, width, device="cuda")
    target = x @ torch.randn(width, width, device="cuda") * width ** -0.5
    losses = [model.step(x, target, k + 1) for k in range(steps)]
    return [v.item() for v in losses], model.forward(x[7:8]), model.forward(x)[7:8]


if __name__ == "__main__":
    losses, one, row = train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    print("loss %.4f -> %.4f in %d steps; one token alone and in the batch differ by %.1e"
          % (losses[0], losses[-1], len(losses), (one.float() - row.float()).abs().max().item()))
