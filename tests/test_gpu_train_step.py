"""examples/train_step.py: the operators together with the merged-gradient path, as a training loop uses them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("grad_dtype", ["bf16", "f16", "f32"])
def test_loss_falls(example, grad_dtype):
    losses = example.train(steps=30, workers=3, tokens=400, hidden=128, grad_dtype=grad_dtype, report=lambda line: print("[train]", line, flush=True))
    assert losses[-1] < 0.5 * losses[0], losses                      # from about log 16


def test_gradients_against_automatic_differentiation(example):
    """Binary32 throughout, so that all that differs is what 8 bits lose: activations are off by at most half a step of 1/127 of
    their channel's largest, so a gradient of weights by about 1/254 of its terms' size, and far less on the whole."""
    net = example.Classifier(hidden=96, inner=160, workers=1, grad_dtype="f32")
    gen = torch.Generator(device="cuda").manual_seed(3)
    ids, types, labels = example.batch(gen, 500, net.shapes[0][0], net.shapes[-1][0])
    loss = net.loss_and_gradients(0, ids, types, labels)
    leaves = [w.detach().double().cpu().requires_grad_(True) for w in net.weights]
    word, position, kind, w1, b1, w2, b2 = leaves
    ids, types, labels = ids.cpu(), types.cpu(), labels.cpu()
    here = (ids >= 0)[:, None]
    h = torch.where(here, word[ids.clamp(min=0)], 0.0) * word.shape[1] ** 0.5 + position[torch.arange(500) % net.length] + kind[types]
    logits = torch.nn.functional.gelu(h @ w1.t() + b1) @ w2.t() + b2
    want = torch.nn.functional.cross_entropy(logits, labels, ignore_index=-1)
    want.backward()
    assert abs(float(loss) - float(want)) < 1e-5 * float(want)
    torch.cuda.synchronize()
    for name, got, leaf in zip(net.names, net.grads[0], leaves):
        off = float((got.double().cpu() - leaf.grad).norm() / leaf.grad.norm())
        print("[train]", name, off, flush=True)
        assert off < (1 / 254 if "weight" in name or name in ("word", "position", "type", "ffn.bias") else 1e-5), (name, off)
    before = [w.clone() for w in net.weights]
    net.update(0.5, 0.9)
    torch.cuda.synchronize()
    for name, w, old, g in zip(net.names, net.weights, before, net.grads[0]):
        assert torch.equal(w, old - 0.5 * g), name                   # one worker, no momentum yet: the gradient itself
    net.close()
