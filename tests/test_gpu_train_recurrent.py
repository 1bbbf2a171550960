"""examples/train_recurrent.py: norm, recurrence and loss together with the operators beside them and the merged-gradient path, as a training loop
uses them; and as an answer is made, token by token."""
import importlib.util
import math
import os

import pytest
import torch

from paper_1912_09268_amd import layers

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_recurrent", os.path.join(ROOT, "examples", "train_recurrent.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("grad_dtype", ["bf16", "f16", "f32"])
def test_it_runs(example, grad_dtype):
    losses = example.train(steps=6, workers=2, sequences=3, length=40, hidden=64, grad_dtype=grad_dtype, report=lambda line: print("[recurrent]", line, flush=True))
    assert len(losses) == 6 and all(math.isfinite(x) for x in losses)


def _reference(net, ids, labels, teacher_ids, teacher, temperature):
    """The same model in 64 bits with automatic differentiation, on the CPU."""
    leaves = {name: w.detach().double().cpu().requires_grad_(True) for name, w in net.weights.items()}
    ids, labels, teacher_ids, teacher = ids.cpu(), labels.cpu().view(-1), teacher_ids.cpu(), teacher.double().cpu()
    sequences, length = ids.shape

    def norm(h, w):
        return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6) * w

    branch = torch.where((ids >= 0)[..., None], leaves["word"][ids.clamp(min=0)], 0.0)
    stream = torch.zeros_like(branch)
    for b in range(net.blocks):
        stream = stream + branch
        z = norm(stream, leaves[f"{b}.norm"]) @ leaves[f"{b}.in.weight"].t() + leaves[f"{b}.in.bias"]
        gate, x = z.split(net.hidden, -1)
        h, out = torch.zeros(sequences, net.hidden, dtype=torch.float64), []
        for t in range(length):
            a = torch.sigmoid(gate[:, t])
            h = a * h + (1 - a) * x[:, t]
            out.append(h)
        branch = torch.stack(out, 1) @ leaves[f"{b}.out.weight"].t()
    logits = (norm(stream + branch, leaves["norm"]) @ leaves["head.weight"].t()).view(sequences * length, -1)
    chosen = labels >= 0
    p = torch.log_softmax(teacher / temperature, 1)
    q = torch.log_softmax(logits / temperature, 1).gather(1, teacher_ids)
    rows = 0.5 * torch.nn.functional.cross_entropy(logits, labels.clamp(min=0), reduction="none") + 0.5 * temperature ** 2 * (p.exp() * (p - q)).sum(1)
    loss = torch.where(chosen, rows, 0.0).sum() / chosen.sum()
    loss.backward()
    return float(loss.detach()), {name: leaf.grad for name, leaf in leaves.items()}


def test_gradients_against_automatic_differentiation(example):
    """Binary32 throughout, so that all that differs is what 8 bits lose: what is kept is off by at most half a step of 1/127 of a channel's largest
    in 128 tokens.  That largest is some three times a channel's root mean square, so what is kept is off by 3 / 254 / sqrt(3) of it in the root
    mean square, errors that do not know of each other; a gradient passes through at most two of them (a norm's, a linear layer's) on each of three
    blocks' ways."""
    net = example.Recurrent(vocabulary=200, hidden=48, blocks=2, workers=1, grad_dtype="f32")
    teacher = example.Teacher(200)
    batch = teacher.batch(torch.Generator(device="cuda").manual_seed(5), 5, 60)
    loss = float(net.loss_and_gradients(0, *batch))
    want, grads = _reference(net, *batch, temperature=2.0)
    assert abs(loss - want) < 1e-5 * want
    torch.cuda.synchronize()
    bound = 3 / 254 / math.sqrt(3) * 2 * 3
    for name in net.names:
        off = float((net.grads[0][name].double().cpu() - grads[name]).norm() / grads[name].norm())
        print("[recurrent]", name, off, flush=True)
        assert off < bound, (name, off)
    before = {name: w.clone() for name, w in net.weights.items()}
    net.update(0.5, 0.9)
    torch.cuda.synchronize()
    for name, w in net.weights.items():
        assert torch.equal(w, before[name] - 0.5 * net.grads[0][name]), name
    net.close()


@pytest.mark.parametrize("grad_dtype", ["bf16", "f32"])
def test_a_captured_step_is_the_eager_one(example, grad_dtype):
    """Forward and backward pass in a HIP graph, replayed on new batches with eager steps between the replays."""
    net = example.Recurrent(vocabulary=200, hidden=64, blocks=2, workers=2, grad_dtype=grad_dtype)
    teacher, gen = example.Teacher(200), torch.Generator(device="cuda").manual_seed(9)
    batch = teacher.batch(gen, 4, 50)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        net.loss_and_gradients(0, *batch)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loss = net.loss_and_gradients(0, *batch)
    for replay in range(4):
        for held, new in zip(batch, teacher.batch(gen, 4, 50)):
            held.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        eager = net.loss_and_gradients(1, *batch)
        torch.cuda.synchronize()
        assert float(loss) == float(eager), replay
        for name in net.names:
            assert torch.equal(net.grads[0][name], net.grads[1][name]), (replay, name)
        net.update(0.1, 0.9)
    net.close()


def test_two_streams_at_once(example):
    """Steps of two workers on two streams, each with its own memory: as one after the other."""
    net = example.Recurrent(vocabulary=300, hidden=128, blocks=2, workers=2, grad_dtype="bf16")
    teacher, gen = example.Teacher(300), torch.Generator(device="cuda").manual_seed(3)
    batches = [teacher.batch(gen, 6, 300) for _ in range(2)]
    want = []
    for k in range(2):
        net.loss_and_gradients(k, *batches[k])
        torch.cuda.synchronize()
        want.append({name: g.clone() for name, g in net.grads[k].items()})
        for g in net.grads[k].values():
            g.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        with torch.cuda.stream(streams[k]):
            net.loss_and_gradients(k, *batches[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(net.grads[k][name], want[k][name]) for name in net.names)
    net.close()


def test_an_answer_token_by_token():
    """The forward pass of a block for one new token of each sequence, its state in place, against the whole sequences at once."""
    g = torch.Generator(device="cuda").manual_seed(8)
    sequences, length, hidden = 3, 30, 64
    weight = 1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")
    into = torch.randn(2 * hidden, hidden, generator=g, device="cuda") * hidden ** -0.5
    x = torch.randn(sequences, length, hidden, generator=g, device="cuda")
    y, _ = layers.norm(x.view(-1, hidden), weight)
    z = (y @ into.t()).view(sequences, length, 2 * hidden)
    whole = layers.recur(z[..., :hidden], z[..., hidden:])
    state = torch.zeros(sequences, hidden, device="cuda")
    for t in range(length):
        y, _ = layers.norm(x[:, t], weight)                              # rows far apart
        z = (y @ into.t()).view(sequences, 1, 2 * hidden)
        out = layers.recur(z[..., :hidden].contiguous(), z[..., hidden:].contiguous(), first=state, last=state)
        assert torch.equal(out[:, 0], state)
        # library products of other sizes: 64 terms of size about 1/8, and what a few tokens of memory make of it
        assert float((state - whole[:, t]).abs().max()) < 64 * 2.0 ** -20
