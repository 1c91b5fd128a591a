"""The operators of a language model's step together: a student's training step (examples/train_student.py) against the same network
in float64 under autograd, captured into graphs, on several streams and threads, far into memory, and the same results every time.

Tolerance of the student's step: every value has passed at most 40 operators in 32 bits, sums of at most 500 products among them:
40 * 500 units of 2^-24 = 1.2e-3, relative to the norm of the tensor.
"""
import importlib.util
import os
import threading

import pytest
import torch

import paper_1801_00829_b200 as fo
from test_gpu_lm import BF16, F16, F32, Distill, Heads, Scan, close, host, ref, unit

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STEP = 40 * 500 * 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_student", os.path.join(ROOT, "examples", "train_student.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_loss(student, w, tokens, positions, reset, ids, values, tail, weight):
    """The student's loss in plain operators."""
    norm = lambda t, g: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * g  # noqa: E731
    x = w["embedding"][tokens]
    y = norm(x, w["norm1"])
    a, v = torch.sigmoid(y @ w["wg"]), y @ w["wx"]
    state, hs = torch.zeros_like(v[:, 0]), []
    for t in range(tokens.shape[1]):
        state = torch.where(reset[:, t, None], 0.0, a[:, t] * state) + (1.0 - a[:, t].square()).sqrt() * v[:, t]
        hs.append(state)
    x = x + torch.stack(hs, 1) @ w["wo"]
    q, k, v = student.split(norm(x, w["norm2"]) @ w["wqkv"])
    cos, sin = (t.double()[positions][:, :, None] for t in (student.cos, student.sin))

    def turn(t):
        b, c = t.chunk(2, -1)
        return torch.cat([b * cos - c * sin, c * cos + b * sin], -1)

    q, k = turn(norm(q, w["q_norm"])), turn(norm(k, w["k_norm"]))
    x = x + student.attend(q, k, v, reset) @ w["wp"]
    z = (norm(x, w["norm3"]) @ w["embedding"].t()).flatten(0, 1).log_softmax(1)
    logp = values.double() - tail.double()[:, None]
    logq = z.gather(1, ids)
    p, left, rest = logp.exp(), 1.0 - logp.exp().sum(1), 1.0 - logq.exp().sum(1)
    return (((p * (logp - logq)).sum(1) + left * (left / rest).log()) * weight.double()).sum()


def test_a_training_step(example):
    torch.manual_seed(3)
    student = example.Student()
    for name in ("norm1", "norm2", "norm3", "q_norm", "k_norm"):
        student.weights[name].data += 0.3 * torch.randn_like(student.weights[name])
    batch = example.batch_of(torch.randn(500, 500, device="cuda"), torch.randint(0, 500, (3, 37), device="cuda"), 16)
    loss = student.loss(*batch)
    loss.backward()
    wide = {n: t.detach().double().requires_grad_() for n, t in student.weights.items()}
    want = plain_loss(student, wide, *batch)
    want.backward()
    assert abs(loss.item() - want.item()) <= STEP * want.item()
    for n, t in student.weights.items():
        assert (t.grad.double() - wide[n].grad).norm() <= STEP * wide[n].grad.norm(), n


def test_token_by_token(example):
    torch.manual_seed(4)
    student = example.Student()
    tokens = torch.randint(0, 500, (25,), device="cuda")
    with torch.no_grad():
        whole = student.logits(tokens[None], torch.arange(25, device="cuda")[None], torch.zeros(1, 25, dtype=torch.bool, device="cuda"))
    assert (student.one_by_one(tokens) - whole).norm() <= STEP * whole.norm()


def test_the_example_runs(example):
    losses, _ = example.train(steps=4)
    assert len(losses) == 4 and all(v == v for v in losses)


# ------------------------------------------------------------------------------------------------------------ graphs, streams, threads
class Step:
    """One call of everything, forwards and backwards; the recurrences in clusters, in chunks and for one token."""

    def __init__(self, seed=0, dtype=BF16):
        self.heads = Heads(2, 75, 6, 2, 64, 64, dtype, bias=True, seed=seed)
        self.scans = [Scan(2, 600, 70, dtype, dtype, "sigmoid", "rest", reset=0.05, seed=seed),
                      Scan(1, 8500, 66, dtype, F32, "exp", "root", reset=0.001, seed=seed), Scan(5, 1, 70, dtype, dtype, "sigmoid", "rest", seed=seed)]
        self.distill = Distill(60, 5001, 20, dtype, True, seed=seed)

    def run(self):
        c = self.heads
        out = list(fo.fused_head_norm(c.q, c.k, **c.how()))
        got = fo.fused_head_norm_grad(c.dq, c.dk, c.q, c.k, **c.how())
        out += [got[k] for k in sorted(got)]
        for c in self.scans:
            h, last = fo.fused_scan(c.x, c.gate, **c.how())
            got = fo.fused_scan_grad(c.dh, c.x, c.gate, h, dlast=c.dlast, **c.how())
            out += [h, last] + [got[k] for k in sorted(got)]
        c = self.distill
        loss, stats = fo.fused_distill(*c.args(), stats=True, **c.how())
        out += [loss, stats, fo.fused_distill_grad(c.dloss, *c.args(), stats, **c.how())]
        return out + list(fo.fused_distill_step(c.dloss, *c.args(), **c.how()))


def same(a, b):
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_the_same_every_time(dtype):
    c = Step(dtype=dtype)
    first = [t.clone() for t in c.run()]
    for _ in range(5):
        assert same(first, c.run())


def test_captured_and_replayed():
    """Two graphs and calls beside them, on the captured stream and others, do not touch each other's scratch."""
    cases = [Step(0), Step(1)]
    want = [[t.clone() for t in c.run()] for c in cases]
    side = torch.cuda.Stream()
    graphs, got = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for c, g in zip(cases, graphs):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            got.append(c.run())
    other = Step(2)
    alone = [t.clone() for t in other.run()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for outs in got:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(side):
            there = other.run()
        torch.cuda.synchronize()
        assert same(there, alone) and same(got[0], want[0]) and same(got[1], want[1])


def test_a_backward_pass_captured_beside_a_living_graph(example):
    """A training step under autograd in a graph, while an eager graph of the same weights lives."""
    torch.manual_seed(5)
    student = example.Student()
    batch = example.batch_of(torch.randn(500, 500, device="cuda"), torch.randint(0, 500, (2, 20), device="cuda"), 8)
    params = list(student.weights.values())
    want = torch.autograd.grad(student.loss(*batch), params)
    living = student.loss(*batch)
    with torch.no_grad():
        leaves = [p.detach().clone().requires_grad_() for p in params]
    eager, student.weights = student.weights, dict(zip(student.weights, leaves))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        torch.autograd.grad(student.loss(*batch), leaves)    # the library's products ask for their workspaces
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = torch.autograd.grad(student.loss(*batch), leaves)
    graph.replay()
    torch.cuda.synchronize()
    # the embedding's gradient is added up by the framework's atomics, in any order
    for n, a, b in zip(eager, got, want):
        assert (a - b).norm() <= STEP * b.norm(), n
    for a, b in zip(torch.autograd.grad(living, params), want):
        assert (a - b).norm() <= STEP * b.norm()


def test_streams_and_threads():
    """Calls at once from four threads with a stream each, and tensors made on another stream than they are used on."""
    cases = [Step(k) for k in range(4)]
    want = [[t.clone() for t in c.run()] for c in cases]
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(4):
                    got[k] = cases[k].run()
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and all(same(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------------------------------------------------ far into memory
FAR = 2 ** 31 + 4096                                         # elements between two rows


def far(shape, dtype, steps):
    """A tensor of `shape` whose indexes lie `steps` elements apart."""
    size = 1 + sum((n - 1) * s for n, s in zip(shape, steps))
    return torch.empty(size, dtype=dtype, device="cuda").as_strided(shape, steps)


def test_strides_beyond_32_bits():
    torch.manual_seed(6)
    c = Heads(2, 3, 2, 1, 64, 64, BF16)
    q = far((2, 3, 2, 64), BF16, (FAR, 128, 64, 1)).copy_(c.q)
    assert same(fo.fused_head_norm(q, c.k, **c.how()), fo.fused_head_norm(c.q, c.k, **c.how()))
    out = far((2, 3, 2, 64), BF16, (FAR, 128, 64, 1))
    fo.fused_head_norm(c.q, c.k, out_q=out, **c.how())
    assert torch.equal(out, fo.fused_head_norm(c.q, c.k, **c.how())[0])
    del q, out
    for tokens, steps in ((3, (2 * FAR, FAR // 2, 1)), (40, (64, 2 ** 27, 1)), (40, (FAR, 64, 1))):
        c = Scan(2, tokens, 64, BF16, BF16, "sigmoid", "rest")
        x = far((2, tokens, 64), BF16, steps)
        x.copy_(c.x)
        want = fo.fused_scan(c.x, c.gate, **c.how())
        assert same(fo.fused_scan(x, c.gate, **c.how()), want)
        a = fo.fused_scan_grad(x, x, c.gate, want[0], **c.how())
        b = fo.fused_scan_grad(c.x, c.x, c.gate, want[0], **c.how())
        assert all(torch.equal(a[k], b[k]) for k in b)
        del x
    c = Distill(3, 1000, 8, BF16, True)
    z = far((3, 1000), BF16, (FAR, 1)).copy_(c.logits)
    want = fo.fused_distill_step(c.dloss, *c.args(), **c.how())
    assert same(fo.fused_distill_step(c.dloss, z, c.ids, c.values, **c.how()), want)
    loss, stats = fo.fused_distill(z, c.ids, c.values, stats=True, **c.how())
    dz = fo.fused_distill_grad(c.dloss, z, c.ids, c.values, stats, out=z, **c.how())
    assert dz is z and torch.allclose(dz.float(), want[1].float(), rtol=2.0 ** -7, atol=2.0 ** -24)


def test_a_long_sequence_of_one_channel():
    """One channel over 2^17 tokens, in as many chunks as there is room for."""
    c = Scan(1, 1 << 17, 1, F32, F32, "sigmoid", "rest", reset=0.0001)
    c.check()


def test_rows_behind_the_last_sequence_stay():
    """A buffer that is larger than the call: what lies around its rows keeps its values."""
    c = Scan(2, 50, 70, BF16, BF16, "sigmoid", "rest", lengths=[50, 20])
    big = torch.full((3, 60, 80), 7.0, dtype=BF16, device="cuda")
    h, _ = fo.fused_scan(c.x, c.gate, out=big[:2, :50, :70], **c.how())
    want, error, _, _ = ref.scan(host(c.x), host(c.gate), **c.host_how())
    close(h, want, unit(BF16) * error, "h")
    assert (big[2] == 7).all() and (big[:, 50:] == 7).all() and (big[:, :, 70:] == 7).all()
    c = Heads(1, 9, 3, 1, 40, 20, F32)
    big = torch.full((10, 3, 48), 7.0, device="cuda")
    fo.fused_head_norm(c.q[0], c.k[0], c.norms[0], c.norms[1], c.rotate[:2] + (c.positions[0],) + c.rotate[3:], out_q=big[:9, :, :40])
    assert (big[9] == 7).all() and (big[:, :, 40:] == 7).all()
    c = Distill(5, 333, 8, F32, False)
    big = torch.full((6, 340), 7.0, device="cuda")
    loss, stats = fo.fused_distill(*c.args(), stats=True, **c.how())
    fo.fused_distill_grad(c.dloss, *c.args(), stats, out=big[:5, :333], **c.how())
    assert (big[5] == 7).all() and (big[:, 333:] == 7).all()
