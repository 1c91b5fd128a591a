"""Trains a small student on a teacher's top logits, then continues a sequence token by token.

    python examples/train_student.py [steps]

The student embeds tokens, passes them through a block with a gated recurrence and a block with attention, and gives logits by
its embedding:  x1 = x + scan(norm(x) Wx, norm(x) Wg) Wo,  x2 = x1 + attention(q, k, v) Wp  with the queries and keys of norm(x1) Wqkv
normed by head and turned by position,  logits = norm(x2) E^T.  The fused operators enter the graph as
autograd.Functions: their backward passes are the operators' own.  The loss's gradient to the logits is there after its forward
pass, which reads them once.  The teacher is a table of random logits for every token and the one before it.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1801_00829_b200 as fo  # noqa: E402

EPS = 1e-6


class Norm(torch.autograd.Function):
    """h = x + f (f None: x), y = norm(h) * weight."""

    @staticmethod
    def forward(ctx, x, f, weight):
        pre = ("rms", weight, None, EPS)
        h, y, stats = fo.fused_block_norm(x, f, pre=pre, stats=True)
        ctx.save_for_backward(h, f, weight, stats)
        return (y, y.new_empty(0)) if f is None else (y, h)

    @staticmethod
    def backward(ctx, dy, dh):
        h, f, weight, stats = ctx.saved_tensors
        got = fo.fused_block_norm_grad(None if f is None else dh.contiguous(), dy.contiguous(), h, f, stats, pre=("rms", weight, None, EPS))
        return got["x"], got.get("f"), got["pre_w"]


class HeadNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions):
        ctx.rotate = (cos, sin, positions, "halves", None)
        ctx.save_for_backward(q, k, q_weight, k_weight)
        return fo.fused_head_norm(q, k, ("rms", q_weight, None, EPS), ("rms", k_weight, None, EPS), ctx.rotate)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, q_weight, k_weight = ctx.saved_tensors
        got = fo.fused_head_norm_grad(dq, dk, q, k, ("rms", q_weight, None, EPS), ("rms", k_weight, None, EPS), ctx.rotate)
        return got["q"], got["k"], got["q_w"], got["k_w"], None, None, None


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, reset):
        h, last = fo.fused_scan(x, gate, "sigmoid", "root", reset=reset)
        ctx.save_for_backward(x, gate, h, reset)
        return h, last

    @staticmethod
    def backward(ctx, dh, dlast):
        x, gate, h, reset = ctx.saved_tensors
        got = fo.fused_scan_grad(dh.contiguous(), x, gate, h, "sigmoid", "root", reset=reset, dlast=dlast.contiguous())
        return got["x"], got["gate"], None


class Distill(torch.autograd.Function):
    """The rows' mean loss; rows without weight are padding."""

    @staticmethod
    def forward(ctx, logits, ids, values, tail, weight):
        loss, dlogits = fo.fused_distill_step(weight, logits, ids, values, tail)
        ctx.save_for_backward(dlogits)
        return (loss * weight).sum()

    @staticmethod
    def backward(ctx, d):
        return ctx.saved_tensors[0] * d, None, None, None, None


class Student:
    SHAPES = dict(embedding=("vocab", "width"), wx=("width", "inner"), wg=("width", "inner"), wo=("inner", "width"),
                  wqkv=("width", "heads"), wp=("attended", "width"), norm1=("width",), norm2=("width",), norm3=("width",),
                  q_norm=("dim",), k_norm=("dim",))

    def __init__(self, vocab=500, width=64, inner=96, heads=4, shared=2, dim=32, length=256, device="cuda"):
        self.heads, self.shared, self.dim = heads, shared, dim
        size = dict(vocab=vocab, width=width, inner=inner, dim=dim, heads=(heads + 2 * shared) * dim, attended=heads * dim)
        self.weights = {}
        for name, shape in self.SHAPES.items():
            shape = [size[s] for s in shape]
            t = torch.randn(shape, device=device) * (shape[1] if name == "embedding" else shape[0]) ** -0.5 if len(shape) == 2 \
                else torch.ones(shape, device=device)
            self.weights[name] = t.requires_grad_()
        angle = torch.arange(length, device=device)[:, None] * 1000.0 ** (-torch.arange(dim // 2, device=device) / (dim // 2))
        self.cos, self.sin = angle.cos(), angle.sin()
        params = list(self.weights.values())
        self.grads = [torch.zeros_like(p) for p in params]
        self.m, self.v = ([torch.zeros_like(p) for p in params] for _ in range(2))
        with torch.no_grad():
            self.norms = fo.tensor_list(self.grads)
            self.update = fo.adam_list(params, self.grads, self.m, self.v)

    def split(self, qkv):
        """(batch, tokens, heads, dim) each, as views of the projection."""
        t = qkv.view(*qkv.shape[:2], -1, self.dim)
        return t.split([self.heads, self.shared, self.shared], 2)

    def logits(self, tokens, positions, reset):
        w, (batch, count) = self.weights, tokens.shape
        x = w["embedding"][tokens]
        y, _ = Norm.apply(x.view(batch * count, -1), None, w["norm1"])
        y = y.view(batch, count, -1)
        h, _ = Scan.apply(y @ w["wx"], y @ w["wg"], reset)
        y, x1 = Norm.apply(x.view(batch * count, -1), (h @ w["wo"]).view(batch * count, -1), w["norm2"])
        q, k, v = self.split((y @ w["wqkv"]).view(batch, count, -1))
        q, k = HeadNorm.apply(q, k, w["q_norm"], w["k_norm"], self.cos, self.sin, positions)
        y, _ = Norm.apply(x1, (self.attend(q, k, v, reset) @ w["wp"]).view(batch * count, -1), w["norm3"])
        return y @ w["embedding"].t()

    def attend(self, q, k, v, reset):
        """Causal, and within a document."""
        document = reset.cumsum(1)
        seen = (document[:, :, None] == document[:, None, :]) & torch.ones(q.shape[1], q.shape[1], dtype=torch.bool, device=q.device).tril()
        q, k, v = (t.transpose(1, 2) for t in (q, k, v))
        k, v = (t.repeat_interleave(self.heads // self.shared, 1) for t in (k, v))
        a = torch.softmax((q @ k.transpose(2, 3) * self.dim ** -0.5).masked_fill(~seen[:, None], float("-inf")), -1)
        return (a @ v).transpose(1, 2).flatten(2)

    def loss(self, tokens, positions, reset, ids, values, tail, weight):
        return Distill.apply(self.logits(tokens, positions, reset), ids, values, tail, weight)

    def step(self, batch, number, lr=1e-2):
        for p in self.weights.values():
            p.grad = None
        loss = self.loss(*batch)
        loss.backward()
        with torch.no_grad():
            for g, p in zip(self.grads, self.weights.values()):
                g.copy_(p.grad)
            result = fo.fused_grad_norm(self.norms, 1.0)
            fo.fused_adamw(self.update, lr=lr, step=number, factor=result[1:])
        return loss.detach()

    @torch.no_grad()
    def one_by_one(self, tokens):
        """Logits of a sequence whose tokens come one after the other: the recurrence's state is handed on, keys and values are kept."""
        w, state, keys, values, rows = self.weights, None, [], [], []
        for t, token in enumerate(tokens):
            x = w["embedding"][token].view(1, -1)
            _, y, _ = fo.fused_block_norm(x, pre=("rms", w["norm1"], None, EPS))
            h, state = fo.fused_scan(y @ w["wx"], y @ w["wg"], "sigmoid", "root", state, out_state=state)
            x, y, _ = fo.fused_block_norm(x, h @ w["wo"], pre=("rms", w["norm2"], None, EPS))
            q, k, v = self.split((y @ w["wqkv"]).view(1, 1, -1))
            at = torch.tensor([[t]], device=x.device)
            q, k = fo.fused_head_norm(q, k, ("rms", w["q_norm"], None, EPS), ("rms", w["k_norm"], None, EPS), (self.cos, self.sin, at, "halves", None))
            keys.append(k[0, 0]), values.append(v[0, 0])
            k, v = (torch.stack(s).repeat_interleave(self.heads // self.shared, 1) for s in (keys, values))
            a = torch.softmax((q[0, 0] * k).sum(2) * self.dim ** -0.5, 0)
            _, y, _ = fo.fused_block_norm(x, (a[:, :, None] * v).sum(0).view(1, -1) @ w["wp"], pre=("rms", w["norm3"], None, EPS))
            rows.append(y @ w["embedding"].t())
        return torch.cat(rows)


def batch_of(teacher, tokens, top, padding=3):
    """Tokens, their positions within documents and the documents' beginnings, the teacher's top logits with its log-sum-exp, weights."""
    batch, count = tokens.shape
    reset = torch.zeros(batch, count, dtype=torch.bool, device=tokens.device)
    reset[:, 0] = reset[::2, count // 3] = True
    place = torch.arange(count, device=tokens.device).expand(batch, -1)
    positions = place - (place * reset).cummax(1).values
    before = torch.where(reset, tokens, tokens.roll(1, 1))
    rows = (teacher[tokens] + 0.5 * teacher[before]).view(batch * count, -1)
    values, ids = rows.topk(top, 1)
    weight = torch.ones(batch, count, device=tokens.device)
    weight[:, count - padding:] = 0.0
    return tokens, positions, reset, ids, values, rows.logsumexp(1), (weight / weight.sum()).view(-1)


def train(steps=80, batch=8, count=48, top=16, seed=0):
    torch.manual_seed(seed)
    student = Student()
    teacher = torch.randn(500, 500, device="cuda") * 2.0
    losses = [student.step(batch_of(teacher, torch.randint(0, 500, (batch, count), device="cuda"), top), k + 1) for k in range(steps)]
    return [v.item() for v in losses], student


if __name__ == "__main__":
    losses, student = train(int(sys.argv[1]) if len(sys.argv) > 1 else 80)
    print("loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], len(losses)))
    tokens = torch.randint(0, 500, (20,), device="cuda")
    reset = torch.zeros(1, 20, dtype=torch.bool, device="cuda")
    with torch.no_grad():
        whole = student.logits(tokens[None], torch.arange(20, device="cuda")[None], reset)
    print("logits token by token and at once differ by %.1e" % (student.one_by_one(tokens) - whole).abs().max().item())
