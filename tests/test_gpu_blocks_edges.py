"""Norm and recurrence where their other tests do not go: teams with several rows and dw, checkpoints side by side, binary16 between offsets, a token whose gate and
value are halves of one product, captured with its state in place."""
import math

import pytest
import torch

from paper_1912_09268_amd import layers
from test_gpu_layers import BF16, DT, G, _close, _gen
from test_gpu_norm import TYPES, _back_reference, _inputs
from test_gpu_recur import CUTS, KINDS, _check, _gate_like, _strided_like

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _say(*a):
    print("[edges]", *a, flush=True)


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("tokens,channels", [(17000, 128), (33000, 100), (5000, 512), (13000, 300), (9000, 1001), (1300, 2048), (2600, 1500), (1300, 4096), (1700, 2100), (1300, 6000)])
def test_teams_that_go_through_several_rows(tokens, channels, dtype, stream):
    """Rows on their way while one is worked on, sums of two rows in turn, scales taken up anew at a group's end within a team's rows, dw of many teams.

    dw: a team adds up to 5 rows, a workgroup up to 64 teams, 32 lanes of the join 16 workgroups each and one of them those 32; a product has two roundings."""
    _say("rows", tokens, channels, dtype, stream)
    g, x, r, w = _inputs(tokens, channels, dtype, stream, "dense", tokens + channels)
    kept = layers.norm_empty(tokens, channels)
    layers.norm(x, w, residual=r, kept=kept)
    dy = torch.randn(tokens, channels, generator=g, device="cuda").to(DT[dtype])
    dres = torch.randn(tokens, channels, generator=g, device="cuda").to(DT[stream])
    dh, dx, dw = torch.empty_like(dres), torch.empty_like(dy), torch.empty(channels, device="cuda")
    layers.norm_backward(kept, dy, w, dres=dres, dh=dh, dx=dx, dw=dw)
    want, off, want_w, _ = _back_reference(kept, dy, w, dres)
    _close(dh, want, off, "dh")
    _close(dx, want, off, "dx")
    n = kept.act.q[:, :channels].double() * kept.act.scale.double().repeat_interleave(G, 0)[:tokens, :channels]
    _close(dw, want_w, (5 + 64 + 16 + 32 + 4) * U * (dy.double() * n).abs().sum(0), "dw")
    rows = dh.clone()
    again = layers.norm_backward(kept, dy, w, dres=dres)                  # without dw: the same rows
    assert torch.equal(again, rows)


@pytest.mark.parametrize("tokens,channels,ld", [(300, 20, 96), (130, 1001, 1040), (40, 16390, 16432)])
def test_checkpoints_side_by_side(tokens, channels, ld):
    """A norm's codes and scales in the columns of a wider memory: those behind its own are left as they are, and not looked at."""
    _say("side by side", tokens, channels, ld)
    g = _gen(ld)
    own = -(-channels // 16) * 16
    x, w = torch.randn(tokens, channels, generator=g, device="cuda"), torch.randn(channels, generator=g, device="cuda")
    kept = layers.norm_empty(tokens, channels)
    y, _ = layers.norm(x, w, kept=kept)
    q = torch.full((tokens, ld), 77, dtype=torch.int8, device="cuda")
    scale, linear = (torch.full((-(-tokens // G), ld), math.nan, device="cuda") for _ in range(2))
    wide = layers.Norm8(layers.Act8(q, scale, channels), torch.empty(tokens, device="cuda"), layers.Act8(q, linear, channels))
    assert torch.equal(layers.norm(x, w, kept=wide)[0], y)
    for narrow, of in ((kept.act.q, q), (kept.act.scale, scale), (kept.linear.scale, linear)):
        assert torch.equal(of[:, :own], narrow[:, :own])
    assert bool((q[:, own:] == 77).all()) and bool(scale[:, own:].isnan().all()) and bool(linear[:, own:].isnan().all())
    dw, dw2 = torch.empty(channels, device="cuda"), torch.empty(channels, device="cuda")
    dh = layers.norm_backward(kept, y, w, dw=dw)
    assert torch.equal(layers.norm_backward(wide, y, w, dw=dw2), dh) and torch.equal(dw2, dw)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cuts", CUTS)
@pytest.mark.parametrize("tokens,channels", [(15, 64), (130, 130), (1000, 41), (5003, 10)])
def test_binary16_between_offsets(tokens, channels, cuts, kind):
    at = CUTS[cuts](tokens)
    _say("packed f16", tokens, channels, cuts, kind)
    g = _gen(tokens + len(at))
    offsets = torch.tensor(at, device="cuda", dtype=torch.int64 if tokens % 2 else torch.int32)
    how = "strided" if channels % 2 else "dense"
    gate = _strided_like(_gate_like((tokens, channels), g).to(DT["f16"]), how)
    x, dy = (_strided_like(torch.randn(tokens, channels, generator=g, device="cuda").to(DT["f16"]), how) for _ in range(2))
    for t in (gate, x, dy):
        t[at[-1]:] = math.nan
    first, dlast = (torch.randn(len(at) - 1, channels, generator=g, device="cuda") for _ in range(2))
    some = len(at) % 2 == 1
    _check(gate, x, kind, first if some else None, dlast if some else None, dy, offsets, at, how)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("length", [1, 5, 20])
@pytest.mark.parametrize("sequences", [1, 9])
def test_gate_and_value_as_halves_of_one_product(sequences, length, dtype):
    """[sequences, length, 2 channels] cut along the last axis, forward and back, into halves of one memory: the bits of tensors by themselves."""
    _say("halves", sequences, length, dtype)
    channels = 72
    g = _gen(sequences + length)
    z = _gate_like((sequences, length, 2 * channels), g).to(DT[dtype])
    gate, x = z[..., :channels], z[..., channels:]
    state = torch.randn(sequences, channels, generator=g, device="cuda")
    states, more = layers.recur_empty(gate), layers.recur_empty(gate)
    first = state.clone()
    y = layers.recur(gate.contiguous(), x.contiguous(), first=first, states=states)
    for out in (None, torch.empty_like(y)):
        last = state.clone()
        got = layers.recur(gate, x, first=last, last=last, states=more, y=out)
        assert torch.equal(got, y) and torch.equal(more, states)
        assert length > 1 or dtype != "f32" or torch.equal(last, y[:, 0])
    dy = torch.randn(y.shape, generator=g, device="cuda").to(DT[dtype])
    dgate, dx = layers.recur_backward(gate.contiguous(), x.contiguous(), states, dy, first=first)
    dz = torch.full_like(z, math.nan)
    layers.recur_backward(gate, x, states, dy, first=first, dgate=dz[..., :channels], dx=dz[..., channels:])
    assert torch.equal(dz[..., :channels], dgate) and torch.equal(dz[..., channels:], dx)


@pytest.mark.parametrize("length", [1, 30, 4099])
def test_a_step_with_its_state_in_place_captured(length):
    """A graph whose state goes in and out in one memory: each replay goes on from where the last one ended, as eager calls do."""
    _say("captured step", length)
    sequences, channels = 2, 40
    g = _gen(length)
    z = torch.zeros(sequences, length, 2 * channels, device="cuda", dtype=BF16)
    state, y = torch.randn(sequences, channels, generator=g, device="cuda"), torch.empty(sequences, length, channels, device="cuda", dtype=BF16)
    eager, held = state.clone(), state.clone()

    def step():
        layers.recur(z[..., :channels], z[..., channels:], kind="unit", first=state, last=state, y=y)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    state.copy_(held)
    for replay in range(4):
        z.copy_(_gate_like(z.shape, g))
        graph.replay()
        torch.cuda.synchronize()
        want = layers.recur(z[..., :channels], z[..., channels:], kind="unit", first=eager, last=eager)
        assert torch.equal(state, eager) and torch.equal(y, want), replay
