"""A small recurrent language model that learns from a teacher's top logits and from labels, on P workers' batches, all on one GPU.

Embedding, blocks of norm -> linear -> gated linear recurrence -> linear with a residual stream, a last norm and an output layer.  Forward and
backward pass are made of the operators of paper_1912_09268_amd.layers and torch's products; what the backward pass needs of the activations is held
in 8 bits, and each worker's gradients are written into the very tensors that group_pipeline packs, averages and applies.

    python examples/train_recurrent.py [--steps 40] [--workers 4] [--sequences 8] [--length 64] [--hidden 128] [--blocks 2] [--grad-dtype bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1912_09268_amd as M  # noqa: E402
from paper_1912_09268_amd import layers  # noqa: E402
from paper_1912_09268_amd.harness import DeviceModel  # noqa: E402

GRAD_DTYPES = {"f32": (torch.float32, M.F32), "bf16": (torch.bfloat16, M.BF16), "f16": (torch.float16, M.F16)}


class Recurrent:
    """Weights, momenta and P workers' gradients in a DeviceModel; forward and backward pass by hand."""

    def __init__(self, vocabulary=600, hidden=128, blocks=2, workers=4, grad_dtype="bf16", seed=0):
        self.names, self.shapes = ["word"], [(vocabulary, hidden)]
        for b in range(blocks):
            self.names += [f"{b}.norm", f"{b}.in.weight", f"{b}.in.bias", f"{b}.out.weight"]
            self.shapes += [(hidden,), (2 * hidden, hidden), (2 * hidden,), (hidden, hidden)]
        self.names += ["norm", "head.weight"]
        self.shapes += [(hidden,), (vocabulary, hidden)]
        self.blocks, self.workers, self.hidden = blocks, workers, hidden
        self.dtype, grad_code = GRAD_DTYPES[grad_dtype]
        sizes = [int(torch.Size(s).numel()) for s in self.shapes]
        itemsize = torch.empty(0, dtype=self.dtype).element_size()
        self.merged, _ = M.plan([n * itemsize for n in sizes], [1e-6 + 1e-10 * n for n in sizes], 2e-5, 1e-10)
        self.ctx = M.Context(sizes, self.merged, workers, grad_code)
        self.model = DeviceModel(self.ctx, sizes)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.weights = {name: w.view(s) for name, w, s in zip(self.names, self.model.w, self.shapes)}
        for name, v in zip(self.names, self.model.v):
            w = self.weights[name]
            if name.endswith("norm"):
                w.fill_(1.0)
            elif name.endswith("bias"):
                w.zero_()
                w[:hidden] = torch.rand(hidden, generator=gen, device="cuda") * 4.0      # gates that remember for a token and for fifty
            else:
                w.normal_(0.0, 1.0 if name == "word" else hidden ** -0.5, generator=gen)
            v.zero_()
        self.grads = [{name: g.view(self.dtype).view(s) for name, g, s in zip(self.names, self.model.grads[k], self.shapes)} for k in range(workers)]

    def loss_and_gradients(self, worker: int, ids: torch.Tensor, labels: torch.Tensor, teacher_ids: torch.Tensor, teacher: torch.Tensor,
                           temperature: float = 2.0, loss_scale: float = 1.0) -> torch.Tensor:
        """One worker's batch: ids and labels [sequences, length] (a place without a label: -1), the teacher's entries [sequences * length, top].
        Gradients, times loss_scale, go to self.grads[worker]; returns the mean loss."""
        grad, hidden = self.grads[worker], self.hidden
        low = {name: w.to(self.dtype) for name, w in self.weights.items() if name.endswith(("weight", "bias"))}
        sequences, length = ids.shape
        tokens = sequences * length

        def split(z):                                    # gate and x of [tokens, 2 hidden], as they lie
            z = z.view(sequences, length, 2 * hidden)
            return z[..., :hidden], z[..., hidden:]

        branch = layers.embed(self.weights["word"], ids.view(-1), dtype=self.dtype)
        stream, memory = None, []
        for b in range(self.blocks):
            kept = layers.norm_empty(tokens, hidden)
            y, stream = layers.norm(branch, self.weights[f"{b}.norm"], residual=stream, kept=kept)
            z = torch.addmm(low[f"{b}.in.bias"], y, low[f"{b}.in.weight"].t())
            gate, x = split(z)
            states = layers.recur_empty(gate)
            r = layers.recur(gate, x, states=states).view(tokens, hidden)
            memory.append((kept, z, states, layers.act_store(r)))
            branch = r @ low[f"{b}.out.weight"].t()
        last = layers.norm_empty(tokens, hidden)
        y, _ = layers.norm(branch, self.weights["norm"], residual=stream, kept=last)
        logits = y @ low["head.weight"].t()
        chosen = labels.view(-1) >= 0
        weight = chosen.float() * (loss_scale / chosen.sum().clamp(min=1))
        loss = layers.distill(logits, teacher_ids, teacher, labels=labels.view(-1), temperature=temperature, label_weight=0.5, teacher_weight=0.5,
                              row_weight=weight, dlogits=logits)
        layers.act_linear_grad(logits, last.linear, grad["head.weight"])
        dh = layers.norm_backward(last, logits @ low["head.weight"], self.weights["norm"], dw=grad["norm"])
        for b in reversed(range(self.blocks)):
            kept, z, states, kept_r = memory[b]
            layers.act_linear_grad(dh, kept_r, grad[f"{b}.out.weight"])
            dr = (dh @ low[f"{b}.out.weight"]).view(sequences, length, hidden)
            dz = torch.empty_like(z)
            layers.recur_backward(*split(z), states, dr, dgate=split(dz)[0], dx=split(dz)[1])
            layers.act_linear_grad(dz, kept.linear, grad[f"{b}.in.weight"], db=grad[f"{b}.in.bias"])
            layers.norm_backward(kept, dz @ low[f"{b}.in.weight"], self.weights[f"{b}.norm"], dres=dh, dh=dh, dw=grad[f"{b}.norm"])
        layers.embed_grad(dh, ids.view(-1), grad["word"])
        return loss.sum() / loss_scale

    def update(self, lr: float, momentum: float) -> None:
        """All workers' gradients packed, averaged and applied in one launch."""
        self.model.group_pipeline(lr, momentum)

    def close(self) -> None:
        self.ctx.close()


class Teacher:
    """A language of pairs: what may follow a word, and how likely.  It is its own best teacher."""

    def __init__(self, vocabulary: int, top: int = 8, seed: int = 1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ids = torch.rand(vocabulary, vocabulary, generator=gen, device="cuda").topk(top, 1).indices
        self.logits = 2.0 * torch.randn(vocabulary, top, generator=gen, device="cuda")

    def batch(self, gen: torch.Generator, sequences: int, length: int):
        """(ids, labels, teacher's ids, teacher's logits); some places behind a sequence's end are padded."""
        words = [torch.randint(0, self.ids.shape[0], (sequences,), generator=gen, device="cuda")]
        for _ in range(length):
            pick = torch.multinomial(torch.softmax(self.logits[words[-1]], 1), 1, generator=gen)
            words.append(self.ids[words[-1]].gather(1, pick).squeeze(1))
        words = torch.stack(words, 1)
        ends = torch.randint(length // 2, length + 1, (sequences, 1), generator=gen, device="cuda")
        padded = torch.arange(length, device="cuda") >= ends
        ids = torch.where(padded, -1, words[:, :-1])
        at = ids.clamp(min=0).view(-1)
        return ids, torch.where(padded, -1, words[:, 1:]), self.ids[at], self.logits[at]


def train(steps=40, workers=4, sequences=8, length=64, hidden=128, blocks=2, grad_dtype="bf16", lr=0.3, momentum=0.9, report=print):
    net = Recurrent(hidden=hidden, blocks=blocks, workers=workers, grad_dtype=grad_dtype)
    teacher = Teacher(net.shapes[0][0])
    gen = torch.Generator(device="cuda").manual_seed(2)
    scale = 256.0 if grad_dtype == "f16" else 1.0
    losses = []
    for step in range(steps):
        losses.append(torch.stack([net.loss_and_gradients(k, *teacher.batch(gen, sequences, length), loss_scale=scale) for k in range(workers)]).mean())
        net.update(lr / scale, momentum)
        if step % 10 == 0 or step == steps - 1:
            report(f"step {step:3d}  loss {float(losses[-1]):.4f}")
    torch.cuda.synchronize()
    net.close()
    return [float(x) for x in losses]


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 40), ("workers", 4), ("sequences", 8), ("length", 64), ("hidden", 128), ("blocks", 2)):
        parser.add_argument(f"--{name}", type=int, default=value)
    parser.add_argument("--grad-dtype", choices=sorted(GRAD_DTYPES), default="bf16")
    a = parser.parse_args()
    train(a.steps, a.workers, a.sequences, a.length, a.hidden, a.blocks, a.grad_dtype)
