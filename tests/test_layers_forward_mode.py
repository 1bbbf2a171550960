"""Tensors with tangents of forward-mode autograd are refused: the operators would lose the tangents without a word."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_1912_09268_amd import layers

OPS = ("embed", "embed_grad", "act_store", "act_backward", "act_linear_grad", "norm", "norm_backward", "recur", "recur_backward", "distill")


def _calls(device):
    """name -> (tensor that is followed, call with it)"""
    t, c = 130, 48
    x, other = torch.randn(t, c, device=device), torch.randn(t, c, device=device)
    w, ids, out = torch.ones(c, device=device), torch.arange(t, device=device) % t, torch.empty(t, c, device=device)
    act, kept = layers.act_empty(t, c, device), layers.norm_empty(t, c, device)
    for m in (act.q, act.scale, kept.act.q, kept.act.scale, kept.rstd, kept.linear.scale):
        m.zero_()
    states = torch.zeros(2, c, device=device)
    loss = torch.empty(t, device=device)
    return {
        "embed": (x, lambda x: layers.embed([x], [ids], out=out)),
        "embed_grad": (x, lambda x: layers.embed_grad(x, ids, out)),
        "act_store": (x, lambda x: layers.act_store(x, act)),
        "act_backward": (x, lambda x: layers.act_backward(act, x, dx=out)),
        "act_linear_grad": (x, lambda x: layers.act_linear_grad(x, act, torch.empty(c, c, device=device))),
        "norm": (w, lambda w: layers.norm(x, w, y=out)),
        "norm_backward": (x, lambda x: layers.norm_backward(kept, x, w, dh=out)),
        "recur": (x, lambda x: layers.recur(other, x, y=out)),
        "recur_backward": (x, lambda x: layers.recur_backward(x, other, states, other, dgate=out, dx=torch.empty_like(out))),
        "distill": (x, lambda x: layers.distill(x, labels=ids % c, loss=loss)),
    }


class Detached(torch.autograd.Function):
    """An operator within a Function that has its own tangent: taken."""
    @staticmethod
    def forward(ctx, x, call):
        call(x)
        return x.clone()

    @staticmethod
    def jvp(ctx, dx, _):
        return dx


def _check(device, takes):
    for name, (x, call) in _calls(device).items():
        print("[forward mode]", name, flush=True)
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(x, torch.ones_like(x))
            for of in (dual, dual.view_as(dual)):
                with pytest.raises(ValueError, match="tangents"):
                    call(of)
                with torch.no_grad(), pytest.raises(ValueError, match="tangents"):
                    call(of)
            if takes:
                call(x)
                call(forward_ad.unpack_dual(dual).primal)
                assert forward_ad.unpack_dual(Detached.apply(dual, call)).tangent is not None
        if takes:
            call(dual)                                                   # behind its level it has no tangent any more


def test_they_are_refused_before_the_device_is_looked_at():
    assert set(_calls("cpu")) == set(OPS)
    _check("cpu", False)


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["native", "plain"])
def test_both_ways(way, monkeypatch):
    if way == "plain":
        for name in OPS:
            monkeypatch.setattr(layers._native, name, lambda *a: NotImplemented)
    _check("cuda", True)
    torch.cuda.synchronize()
