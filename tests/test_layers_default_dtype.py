"""Memory that the operators make is of its own type, whatever torch's default type is."""
import pytest
import torch

from paper_1912_09268_amd import layers


@pytest.fixture(params=[torch.bfloat16, torch.float16, torch.float64])
def default(request):
    before = torch.get_default_dtype()
    torch.set_default_dtype(request.param)
    yield request.param
    torch.set_default_dtype(before)


def test_memory_for_checkpoints_and_states_is_binary32(default):
    kept = layers.norm_empty(130, 20, "cpu")
    assert {t.dtype for t in (layers.act_empty(5, 3, "cpu").scale, kept.rstd, kept.act.scale, kept.linear.scale)} == {torch.float32}
    assert kept.act.q.dtype == torch.int8
    assert layers.recur_empty(torch.zeros(2, 300, 8, dtype=torch.bfloat16)).dtype == torch.float32


@pytest.mark.gpu
def test_operators_under_another_default(default):
    print("[layers] default", default, flush=True)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w = torch.randn(130, 48, generator=g, device="cuda", dtype=torch.float32).bfloat16(), torch.ones(48, device="cuda", dtype=torch.float32)
    kept = layers.norm_empty(130, 48)
    y, _ = layers.norm(x, w, kept=kept)
    dh = layers.norm_backward(kept, y, w)
    act = layers.act_store(x)
    states = layers.recur_empty(x)
    r = layers.recur(x, y, states=states)
    grads = layers.recur_backward(x, y, states, r)
    loss = layers.distill(x, labels=torch.arange(130, device="cuda") % 48)
    assert loss.dtype == act.scale.dtype == torch.float32 and {t.dtype for t in (y, dh, r, *grads)} == {torch.bfloat16}
    torch.set_default_dtype(torch.float32)
    again = layers.norm_empty(130, 48)
    assert torch.equal(layers.norm(x, w, kept=again)[0], y) and torch.equal(again.act.scale, kept.act.scale)
    assert torch.equal(layers.distill(x, labels=torch.arange(130, device="cuda") % 48), loss)
