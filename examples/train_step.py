"""A training loop in which every gradient that the merged-gradient path packs, reduces and applies is made by the operators of
paper_1912_09268_amd.layers.

A small text classifier -- embedding (word + position + type), a feed-forward layer with GELU, an output layer -- on P workers'
batches, all on one GPU.  What the backward pass needs of the activations is held in 8 bits.  Each worker's gradients are written into
the very tensors that group_pipeline reads; the plan, the merge buffers and the SGD-momentum update are the library's.

    python examples/train_step.py [--steps 40] [--workers 4] [--tokens 512] [--hidden 256] [--grad-dtype bf16]
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


class Classifier:
    """Weights, momenta and P workers' gradients in a DeviceModel; forward and backward pass by hand."""

    def __init__(self, vocabulary=1000, length=64, hidden=256, inner=512, classes=16, workers=4, grad_dtype="bf16", seed=0):
        self.shapes = [(vocabulary, hidden), (length, hidden), (2, hidden), (inner, hidden), (inner,), (classes, inner), (classes,)]
        self.names = ["word", "position", "type", "ffn.weight", "ffn.bias", "out.weight", "out.bias"]
        self.length, self.workers = length, workers
        self.dtype, grad_code = GRAD_DTYPES[grad_dtype]
        sizes = [int(torch.Size(s).numel()) for s in self.shapes]
        itemsize = torch.empty(0, dtype=self.dtype).element_size()
        # backward times by size, and a cost model under which some layers are merged
        self.merged, _ = M.plan([n * itemsize for n in sizes], [1e-6 + 1e-10 * n for n in sizes], 2e-5, 1e-10)
        self.ctx = M.Context(sizes, self.merged, workers, grad_code)
        self.model = DeviceModel(self.ctx, sizes)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.weights = [w.view(s) for w, s in zip(self.model.w, self.shapes)]
        for name, w, v in zip(self.names, self.weights, self.model.v):
            w.normal_(0.0, 0.05 if w.dim() > 1 else 0.0, generator=gen)
            v.zero_()
        # the gradients as matrices of their type: the model holds 16-bit ones as raw bits
        self.grads = [[g.view(self.dtype).view(s) for g, s in zip(self.model.grads[k], self.shapes)] for k in range(workers)]

    def loss_and_gradients(self, worker: int, ids: torch.Tensor, types: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        """One worker's batch: ids, types and labels [tokens].  Its gradients go to self.grads[worker]."""
        word, position, kind, w1, b1, w2, b2 = self.weights
        grad = dict(zip(self.names, self.grads[worker]))
        tokens, hidden = ids.numel(), word.shape[1]
        places = torch.arange(tokens, device=ids.device) % self.length
        scale = hidden ** 0.5
        # forward: binary32 master weights, activations of the gradients' type
        low = [w.to(self.dtype) for w in (w1, b1, w2, b2)]
        h = layers.embed([word, position, kind], [ids, places, types], scales=[scale, 1.0, 1.0], dtype=self.dtype)
        kept_h = layers.act_store(h)
        z = torch.addmm(low[1], h, low[0].t())
        u = torch.empty_like(z)
        kept_z = layers.act_store(z, kind="gelu", y=u)               # z in 8 bits and gelu(z) in one pass
        kept_u = layers.act_store(u)
        logits = torch.addmm(low[3], u, low[2].t()).float()
        chosen = labels >= 0                                         # places without a label have no loss
        count = chosen.sum().clamp(min=1)
        p = torch.log_softmax(logits, 1)
        loss = -torch.where(chosen, p.gather(1, labels.clamp(min=0)[:, None]).squeeze(1), 0.0).sum() / count
        # backward
        d = p.exp()
        d.scatter_add_(1, labels.clamp(min=0)[:, None], torch.full((tokens, 1), -1.0, device=d.device))
        d = (torch.where(chosen[:, None], d, 0.0) / count).to(self.dtype)
        layers.act_linear_grad(d, kept_u, grad["out.weight"], db=grad["out.bias"])
        dz = layers.act_backward(kept_z, d @ low[2], kind="gelu")
        layers.act_linear_grad(dz, kept_h, grad["ffn.weight"], db=grad["ffn.bias"])
        dh = dz @ low[0]
        layers.embed_grad(dh, ids, grad["word"], scale=scale)
        layers.embed_grad(dh, places, grad["position"])
        layers.embed_grad(dh, types, grad["type"])
        return loss

    def update(self, lr: float, momentum: float) -> None:
        """All workers' gradients packed, averaged and applied in one launch."""
        self.model.group_pipeline(lr, momentum)

    def close(self) -> None:
        self.ctx.close()


def batch(gen: torch.Generator, tokens: int, vocabulary: int, classes: int):
    """Words of a frequency, some places padded (id -1, no label); a word's class is its number's."""
    u = torch.rand(tokens, generator=gen, device="cuda")
    ids = (torch.exp(u * torch.log(torch.tensor(vocabulary + 1.0, device="cuda"))) - 1).long().clamp(0, vocabulary - 1)
    padded = torch.rand(tokens, generator=gen, device="cuda") < 0.1
    labels = torch.where(padded, -1, ids % classes)
    return torch.where(padded, -1, ids), torch.randint(0, 2, (tokens,), generator=gen, device="cuda"), labels


def train(steps=40, workers=4, tokens=512, hidden=256, grad_dtype="bf16", lr=0.2, momentum=0.9, report=print):
    net = Classifier(hidden=hidden, inner=2 * hidden, workers=workers, grad_dtype=grad_dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for step in range(steps):
        losses.append(torch.stack([net.loss_and_gradients(k, *batch(gen, tokens, net.shapes[0][0], net.shapes[-1][0])) for k in range(workers)]).mean())
        net.update(lr, momentum)
        if step % 10 == 0 or step == steps - 1:
            report(f"step {step:3d}  loss {float(losses[-1]):.4f}")
    torch.cuda.synchronize()
    net.close()
    return [float(x) for x in losses]


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=40)
    parser.add_argument("--workers", type=int, default=4)
    parser.add_argument("--tokens", type=int, default=512)
    parser.add_argument("--hidden", type=int, default=256)
    parser.add_argument("--grad-dtype", choices=sorted(GRAD_DTYPES), default="bf16")
    a = parser.parse_args()
    train(a.steps, a.workers, a.tokens, a.hidden, a.grad_dtype)
