"""The gated linear recurrence and its way back against a plain 64-bit loop over the tokens.

Tolerances, u = 2^-24: a gate's smaller share is off by e = 1.2e-7 |gate| + 3e-7 of itself, the larger one by 3e-7, c by about as much, a step adds two
roundings, whichever way steps are composed (a product of steps has the sum of their relative errors).  So an error bound follows the recurrence
itself: E[t] = a E[t-1] + (e + 4 u) * (a H[t-1] + c |x|), H the recurrence of magnitudes; twice that for a step's going in twice."""
import math

import pytest
import torch

from paper_1912_09268_amd import layers_binding as M
from paper_1912_09268_amd import layers
from test_gpu_layers import BF16, DT, F16, F32, _close, _gen, _strided, _untouched

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
KINDS = ["free", "convex", "unit"]
BLOCK = 128


def _say(*a):
    print("[recur]", *a, flush=True)


def _gates(gate, kind):
    """(a, c, dc/da * da/dgate, error of a, error of c) in 64 bits; errors relative."""
    a, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    small = 1.2e-7 * gate.abs() + 3e-7
    e_a, e_rest = torch.where(gate < 0, small, 3e-7), torch.where(gate < 0, 3e-7, small)
    if kind == "free":
        return a, torch.ones_like(a), torch.zeros_like(a), e_a, torch.zeros_like(a), e_rest
    if kind == "convex":
        return a, rest, -a * rest, e_a, e_rest, e_rest
    return a, torch.sqrt(rest * (1 + a)), -a * a * torch.sqrt(rest / (1 + a)), e_a, e_rest + e_a + 4 * U, e_rest


def _one(gate, x, first, dy, dlast, kind):
    """A sequence [tokens, channels] (or several side by side, [tokens, sequences, channels]) -> a dict of results and slacks."""
    a, c, dc, e_a, e_c, e_rest = _gates(gate, kind)
    tokens = gate.shape[0]
    h, H, E = first.clone(), first.abs(), torch.zeros_like(first)
    out = {k: torch.zeros_like(gate) for k in ("y", "y_off", "before", "before_H", "before_E", "dx", "dx_off", "dgate", "dgate_off")}
    for t in range(tokens):
        out["before"][t], out["before_H"][t], out["before_E"][t] = h, H, E
        step = a[t] * H + c[t] * x[t].abs()
        E = a[t] * E + 2 * ((e_a[t] + 4 * U) * a[t] * H + (e_c[t] + 4 * U) * c[t] * x[t].abs())
        h, H = a[t] * h + c[t] * x[t], step
        out["y"][t], out["y_off"][t] = h, E
    out["last"], out["last_off"] = h, E
    d, D, E = dlast.clone(), dlast.abs(), torch.zeros_like(dlast)
    for t in reversed(range(tokens)):
        d, D, E = dy[t] + d, dy[t].abs() + D, E + 2 * U * (dy[t].abs() + D)
        out["dx"][t], out["dx_off"][t] = c[t] * d, c[t] * (E + (e_c[t] + 4 * U) * D)
        rest = torch.sigmoid(-gate[t])
        slope = a[t] * rest * out["before"][t] + dc[t] * x[t]
        size = a[t] * rest * out["before_H"][t] + dc[t].abs() * x[t].abs()
        slope_off = size * (e_a[t] + e_rest[t] + e_c[t] + 12 * U) + a[t] * rest * out["before_E"][t]
        out["dgate"][t], out["dgate_off"][t] = d * slope, E * size + D * slope_off
        E = a[t] * E + 2 * (e_a[t] + 4 * U) * a[t] * D
        d, D = a[t] * d, a[t] * D
    out["dfirst"], out["dfirst_off"] = d, E
    return out


def _reference(gate, x, first, dy, dlast, kind, cuts):
    """Sequences by the rows between cuts, all in 64 bits on the CPU."""
    gate, x, first, dy, dlast = (t.double().cpu() for t in (gate, x, first, dy, dlast))
    tokens, channels = gate.shape
    rows = ("y", "y_off", "before", "dx", "dx_off", "dgate", "dgate_off")
    total = {k: torch.zeros(tokens, channels, dtype=torch.float64) for k in rows}
    ends = {k: torch.zeros(len(cuts) - 1, channels, dtype=torch.float64) for k in ("last", "last_off", "dfirst", "dfirst_off")}
    lengths = {b - a for a, b in zip(cuts, cuts[1:])}
    for n in lengths:                                                    # those of one length side by side
        of = [i for i in range(len(cuts) - 1) if cuts[i + 1] - cuts[i] == n]
        at = torch.tensor([list(range(cuts[i], cuts[i + 1])) for i in of], dtype=torch.int64).view(len(of), n).t()
        got = _one(gate[at], x[at], first[of], dy[at], dlast[of], kind)
        for k in rows:
            total[k][at] = got[k]
        for k in ends:
            ends[k][of] = got[k]
    return {k: v.cuda() for k, v in {**total, **ends}.items()}


def _gate_like(shape, g):
    """Gates that forget at once, in a few tokens, in hundreds, and not at all."""
    channels = shape[-1]
    at = torch.rand(channels, generator=g, device="cuda") * 10.0 - 2.0
    return torch.randn(shape, generator=g, device="cuda") + at


def _check(gate, x, kind, first, dlast, dy, offsets, cuts, how):
    """All of a forward and a way back: gate, x, dy as the call takes them; cuts: rows of the sequences."""
    channels = gate.shape[-1]
    flat = [t.reshape(-1, channels) for t in (gate, x, dy)]
    sequences = len(cuts) - 1
    zero = torch.zeros(sequences, channels, device="cuda")
    want = _reference(flat[0], flat[1], zero if first is None else first, flat[2], zero if dlast is None else dlast, kind, cuts)
    inside = cuts[-1]

    def like(t):
        if how == "dense" or t.dim() == 3 and t.shape[1] == 1:
            return torch.full_like(t, math.nan, memory_format=torch.contiguous_format), None
        m, whole = _strided((t.numel() // channels, channels), t.dtype, how)
        return (m if t.dim() == 2 else torch.as_strided(m, t.shape, (t.shape[1] * m.stride(0), m.stride(0), 1), m.storage_offset())), (m, whole)

    y, y_whole = like(x)
    last, states = torch.full((sequences, channels), math.nan, device="cuda"), layers.recur_empty(gate, offsets).fill_(math.nan)
    assert layers.recur(gate, x, kind=kind, first=first, offsets=offsets, y=y, last=last, states=states) is y
    rows = y.reshape(-1, channels)
    _close(rows[:inside], want["y"][:inside], want["y_off"][:inside], "y")
    assert bool(rows[inside:].isnan().all())
    assert y_whole is None or _untouched(*y_whole, math.nan)
    _close(last, want["last"], want["last_off"], "last")
    before = want["before"]
    if offsets is not None:
        kept = torch.arange(0, flat[0].shape[0], BLOCK, device="cuda")
        kept = kept[kept < inside]
        _close(states[:kept.numel()], before[kept], 1e-6 + want["y_off"][(kept - 1).clamp(min=0)], "states")
        assert bool(states[kept.numel():].isnan().all())
    elif states.numel():
        length = flat[0].shape[0] // sequences
        kept = torch.cat([torch.arange(s * length, (s + 1) * length, BLOCK, device="cuda") for s in range(sequences)])
        _close(states, before[kept], 1e-6 + want["y_off"][(kept - 1).clamp(min=0)], "states")
    # y alone, nothing else asked for: the same bits
    alone = layers.recur(gate, x, kind=kind, first=first, offsets=offsets)
    assert torch.equal(alone.reshape(-1, channels)[:inside], rows[:inside])
    if first is not None and offsets is None:                            # the state in place
        state = first.clone()
        layers.recur(gate, x, kind=kind, first=state, last=state)
        assert torch.equal(state, last)
    (dgate, g_whole), (dx, x_whole) = like(x), like(x)
    dfirst = torch.full((sequences, channels), math.nan, device="cuda")
    got = layers.recur_backward(gate, x, states, dy, kind=kind, first=first, offsets=offsets, dlast=dlast, dgate=dgate, dx=dx, dfirst=dfirst)
    assert got[0] is dgate and got[1] is dx
    for t, name in ((dgate, "dgate"), (dx, "dx")):
        rows = t.reshape(-1, channels)
        _close(rows[:inside], want[name][:inside], want[name + "_off"][:inside] + 1e-37, name)
        assert bool(rows[inside:].isnan().all())
    _close(dfirst, want["dfirst"], want["dfirst_off"] + 1e-37, "dfirst")
    assert x_whole is None or (_untouched(*x_whole, math.nan) and _untouched(*g_whole, math.nan))
    again = layers.recur_backward(gate, x, states, dy, kind=kind, first=first, offsets=offsets, dlast=dlast)
    for a, b in zip(again, (dgate, dx)):
        assert torch.equal(a.reshape(-1, channels)[:inside], b.reshape(-1, channels)[:inside])
    if offsets is not None:
        assert not bool(again[0][inside:].any()) and not bool(alone[inside:].any())


def _strided_like(t, how):
    if how == "dense":
        return t.contiguous()
    channels = t.shape[-1]
    m, _ = _strided((t.numel() // channels, channels), t.dtype, how)
    m.copy_(t.reshape(-1, channels))
    if t.dim() == 2:
        return m
    return torch.as_strided(m, t.shape, (t.shape[1] * m.stride(0), m.stride(0), 1), m.storage_offset())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sequences,length,channels", [(1, 1, 1), (8, 1, 1024), (3, 2, 7), (5, 16, 130), (4, 17, 65), (2, 127, 64), (2, 128, 129), (3, 129, 33), (1, 500, 200), (2, 1000, 24), (3, 4, 70), (300, 5, 40), (77, 13, 64), (50, 63, 20), (41, 64, 130),
                                                       (700, 20, 9), (1, 4099, 16), (600, 130, 5), (2, 300, 1), (5, 6, 130), (9, 7, 33), (40, 8, 65), (40, 9, 65)])
def test_sequences_of_one_length(sequences, length, channels, kind, dtype):
    how = "strided" if (length + channels) % 2 else "dense"
    _say("one length", sequences, length, channels, kind, dtype, how)
    g = _gen(sequences + length + channels)
    shape = (sequences, length, channels)
    gate = _strided_like(_gate_like(shape, g).to(DT[dtype]), how)
    x = _strided_like(torch.randn(shape, generator=g, device="cuda").to(DT[dtype]), how)
    dy = _strided_like(torch.randn(shape, generator=g, device="cuda").to(DT[dtype]), how)
    first, dlast = (torch.randn(sequences, channels, generator=g, device="cuda") for _ in range(2))
    some = (sequences + length) % 2 == 0 or length == 1
    _check(gate, x, kind, first if some else None, dlast if some else None, dy, None, [s * length for s in range(sequences + 1)], how)


CUTS = {"one": lambda n: [0, n], "two": lambda n: [0, n // 3, n], "empty ones": lambda n: [0, 0, 0, n // 2, n // 2, n, n], "behind": lambda n: [0, n // 5, n // 2],
        "ones": lambda n: list(range(min(n, 300) + 1)), "at blocks": lambda n: sorted({0, min(16, n), min(128, n), min(256, n), n}),
        "many": lambda n: sorted([0, n] + [(i * 7919) % (n + 1) for i in range(min(n, 700))]), "no tokens": lambda n: [0, 0, 0]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cuts", CUTS)
@pytest.mark.parametrize("tokens,channels", [(1, 3), (15, 64), (130, 130), (1000, 40), (5003, 9)])
def test_sequences_one_behind_the_other(tokens, channels, cuts, kind, dtype):
    _say("packed", tokens, channels, cuts, kind, dtype)
    at = CUTS[cuts](tokens)
    g = _gen(tokens + len(at))
    offsets = torch.tensor(at, device="cuda", dtype=torch.int32 if tokens % 2 else torch.int64)
    how = "strided" if channels % 2 else "dense"
    gate = _strided_like(_gate_like((tokens, channels), g).to(DT[dtype]), how)
    x = _strided_like(torch.randn(tokens, channels, generator=g, device="cuda").to(DT[dtype]), how)
    dy = _strided_like(torch.randn(tokens, channels, generator=g, device="cuda").to(DT[dtype]), how)
    for t in (gate, x, dy):
        t[at[-1]:] = math.nan                                            # no sequence's: not looked at
    first, dlast = (torch.randn(len(at) - 1, channels, generator=g, device="cuda") for _ in range(2))
    some = len(at) % 2 == 0
    _check(gate, x, kind, first if some else None, dlast if some else None, dy, offsets, at, how)


def test_more_sequences_than_a_wavefront_searches_at_once():
    tokens, channels = 20000, 8
    for count in (63, 64, 65, 4095, 5000, 19999):
        _say("packed", count)
        g = _gen(count)
        at = [0] + torch.randint(0, tokens + 1, (count - 1,), generator=torch.Generator().manual_seed(count)).sort().values.tolist() + [tokens - 3]
        at = [min(a, tokens - 3) for a in at]
        gate, x, dy = _gate_like((tokens, channels), g), torch.randn(tokens, channels, generator=g, device="cuda"), torch.randn(tokens, channels, generator=g, device="cuda")
        first, dlast = (torch.randn(count, channels, generator=g, device="cuda") for _ in range(2))
        _check(gate, x, "convex", first, dlast, dy, torch.tensor(at, device="cuda"), at, "dense")


@pytest.mark.parametrize("packed", [False, True])
def test_infinities_and_nans_stay_in_their_sequences_and_channels(packed):
    _say("not finite", packed)
    sequences, length, channels = 6, 300, 40
    g = _gen(7)
    gate, x = torch.randn(sequences, length, channels, generator=g, device="cuda"), torch.randn(sequences, length, channels, generator=g, device="cuda")
    gate[0, 0, 0], gate[1, 7, 1], x[2, 290, 2], x[3, 299, 3], x[4, 0, 4] = math.nan, math.inf, math.inf, math.nan, math.inf
    gate[4, 150, 4] = -math.inf                                          # a = 0 does not take an infinity away
    dy = torch.randn(sequences, length, channels, generator=g, device="cuda")
    dy[5, 100, 5] = math.nan
    shape = (sequences * length, channels) if packed else (sequences, length, channels)
    offsets = torch.arange(sequences + 1, device="cuda") * length if packed else None
    gate, x, dy = gate.view(shape), x.view(shape), dy.view(shape)
    states = layers.recur_empty(gate, offsets)
    last = torch.empty(sequences, channels, device="cuda")
    y = layers.recur(gate, x, offsets=offsets, last=last, states=states).view(sequences, length, channels)
    torch.cuda.synchronize()
    fine = torch.ones(sequences, length, channels, dtype=torch.bool, device="cuda")
    fine[0, :, 0] = fine[2, 290:, 2] = fine[3, 299, 3] = fine[4, :, 4] = False
    assert torch.equal(y.isfinite(), fine)
    assert bool((y[2, 290:, 2] == math.inf).all()) and bool(y[4, 150:, 4].isnan().all()) and bool((y[4, :150, 4] == math.inf).all())
    assert torch.equal(last.isfinite(), fine[:, -1])
    dgate, dx = (t.view(sequences, length, channels) for t in layers.recur_backward(gate, x, states, dy, offsets=offsets))
    assert bool(dx[5, :101, 5].isnan().all()) and bool(dx[5, 101:, 5].isfinite().all()) and bool(dx[1:5, :, 6:].isfinite().all()) and bool(dgate[:, :, 6:].isfinite().all())
    assert bool(dx[0, :, 1:].isfinite().all()) and bool(dgate[4, :, 5].isfinite().all())


@pytest.mark.parametrize("offsets", [[5, 3, 9], [0, 1000, 20], [-7, 2 ** 40, 4], [900, 900, 900], [0, -1, -5]])
def test_offsets_that_are_wrong_lead_nowhere_else(offsets):
    """They are kept within the tokens: what comes out says nothing, but nothing else is written."""
    _say("wrong offsets", offsets)
    tokens, channels = 600, 70
    offs = torch.tensor(offsets, device="cuda")
    whole = torch.full((3, tokens, channels), 7.0, device="cuda")
    gate, x = torch.randn(tokens, channels, device="cuda"), torch.randn(tokens, channels, device="cuda")
    first, last = torch.randn(4, channels, device="cuda"), torch.full((4, channels), 7.0, device="cuda")
    states = torch.zeros(layers.recur_empty(gate, offs).shape[0] + 1, channels, device="cuda")
    layers.recur(gate, x, first=first[:2], offsets=offs, y=whole[1], last=last[1:3], states=states[:-1])
    layers.recur_backward(gate, x, states[:-1], x, first=first[:2], offsets=offs, dgate=whole[1], dx=torch.empty_like(x), dfirst=last[1:3])
    torch.cuda.synchronize()
    assert bool((whole[0] == 7).all()) and bool((whole[2] == 7).all()) and bool((last[0] == 7).all()) and bool((last[3] == 7).all()) and not bool(states[-1].any())


def test_sequences_without_tokens_or_channels():
    first = torch.randn(3, 8, device="cuda")
    last, dfirst = torch.empty(3, 8, device="cuda"), torch.empty(3, 8, device="cuda")
    none = torch.empty(3, 0, 8, device="cuda")
    states = layers.recur_empty(none)
    assert states.shape == (0, 8) and layers.recur(none, none, first=first, last=last, states=states).shape == none.shape
    assert torch.equal(last, first)
    layers.recur(none, none, last=last)
    assert not bool(last.any())
    layers.recur_backward(none, none, states, none, dlast=first, dfirst=dfirst)
    assert torch.equal(dfirst, first)
    for shape in ((0, 5, 8), (3, 5, 0), (0, 8), (5, 0)):
        t = torch.empty(shape, device="cuda")
        states = layers.recur_empty(t)
        assert layers.recur(t, t, states=states).shape == shape
        assert layers.recur_backward(t, t, states, t)[0].shape == shape
    offsets = torch.zeros(1, dtype=torch.int64, device="cuda")           # no sequence at all
    t = torch.randn(7, 8, device="cuda")
    assert not bool(layers.recur(t, t, offsets=offsets).any())


def test_step_by_step_is_the_whole():
    """An answer's tokens one by one, the state going in and out in place, against all at once."""
    g = _gen(3)
    sequences, length, channels = 3, 40, 72
    gate, x = _gate_like((sequences, length, channels), g), torch.randn(sequences, length, channels, generator=g, device="cuda")
    whole = layers.recur(gate, x, kind="unit")
    state = torch.zeros(sequences, channels, device="cuda")
    for t in range(length):
        y = layers.recur(gate[:, t:t + 1].contiguous(), x[:, t:t + 1].contiguous(), kind="unit", first=state, last=state)
        assert torch.equal(y[:, 0], state)
        # two ways to the same: both within the bound of the reference, which is below 4e-6 of sizes of a few
        assert float((state - whole[:, t]).abs().max()) < 2e-5


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_against_differences(kind):
    """Along a direction, in 64 bits by the plain loop: the slope against the kernel's gradients."""
    g = _gen(11)
    n, channels = 150, 6
    gate, x, c = (torch.randn(n, channels, generator=g, device="cuda") for _ in range(3))
    first, cl = (torch.randn(1, channels, generator=g, device="cuda") for _ in range(2))
    states, dfirst = layers.recur_empty(gate), torch.empty(1, channels, device="cuda")
    layers.recur(gate, x, kind=kind, first=first, states=states)
    dgate, dx = layers.recur_backward(gate, x, states, c, kind=kind, first=first, dlast=cl, dfirst=dfirst)

    def loss(gate, x, first):
        a, cc, *_ = _gates(gate, kind)
        h, total = first, 0.0
        for t in range(n):
            h = a[t] * h + cc[t] * x[t]
            total += float((h * c64[t]).sum())
        return total + float((h * cl64).sum())

    gate64, x64, first64, c64, cl64 = (t.double().cpu() for t in (gate, x, first[0], c, cl[0]))
    gen = torch.Generator().manual_seed(5)
    for _ in range(3):
        u, v, w = (torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in (gate64, x64, first64))
        e = 1e-5
        along = (loss(gate64 + e * u, x64 + e * v, first64 + e * w) - loss(gate64 - e * u, x64 - e * v, first64 - e * w)) / (2 * e)
        got = float((dgate.double().cpu() * u).sum() + (dx.double().cpu() * v).sum() + (dfirst[0].double().cpu() * w).sum())
        size = float((dgate.double().cpu() * u).abs().sum() + (dx.double().cpu() * v).abs().sum()) + 1
        assert abs(along - got) < 1e-5 * size


def test_offsets_beyond_32_bits():
    _say("offsets beyond 2^32 elements")
    rows, stride, channels = 530000, 8192, 20
    memory = torch.zeros(rows * stride, dtype=BF16, device="cuda")
    x = torch.as_strided(memory, (rows, channels), (stride, 1))
    x[-300:] = torch.randn(300, channels, generator=_gen(1), device="cuda").to(BF16)
    gate = torch.full((rows, channels), -1.0, dtype=BF16, device="cuda")
    states, last = layers.recur_empty(gate), torch.empty(1, channels, device="cuda")
    y = layers.recur(gate, x, last=last, states=states)
    small = layers.recur(gate[-300:], x[-300:].contiguous())
    # zeros before them: exactly the same steps, cut at other places; a = 0.27 forgets a rounding at once
    assert float((y[-300:].double() - small.double()).abs().max()) < 2.0 ** -7
    far = torch.as_strided(memory, (rows, channels), (stride, 1), 4096)                          # dx beyond 32 bits, too
    dgate, dx = layers.recur_backward(gate, x, states, y, dgate=torch.empty_like(y), dx=far)
    near = layers.recur_backward(gate, x.contiguous(), states, y)
    assert torch.equal(dx, near[1]) and torch.equal(dgate, near[0]) and bool(dx[-300:].any())


def test_workspaces_and_graphs():
    """Two captured graphs, the workspace given and torch's own, replayed with eager work between."""
    g = _gen(19)
    n, channels = 3000, 64
    gate, x, dy = (torch.randn(n, channels, generator=g, device="cuda").to(BF16) for _ in range(3))
    offsets = torch.tensor([0, 700, 701, 2990], device="cuda")
    sequences = M.Sequences(3, n, offsets.data_ptr(), M.I64)
    size = M.recur_workspace(sequences, channels, M.BF16)
    assert size > 0
    space = torch.empty(size, dtype=torch.uint8, device="cuda")
    y, last, states = torch.zeros_like(x), torch.empty(3, channels, device="cuda"), layers.recur_empty(gate, offsets)
    dgate, dx, dfirst = torch.zeros_like(x), torch.zeros_like(x), torch.empty(3, channels, device="cuda")
    outs = (y, last, states, dgate, dx, dfirst)

    def forth(space=space):
        layers.recur(gate, x, first=dlast, offsets=offsets, y=y, last=last, states=states, workspace=space)

    def back(space=space):
        layers.recur_backward(gate, x, states, dy, first=dlast, offsets=offsets, dlast=dlast, dgate=dgate, dx=dx, dfirst=dfirst, workspace=space)

    dlast = torch.randn(3, channels, generator=g, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        forth(), back()
    stream.synchronize()
    graphs = []
    for call in (forth, back):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            call()
    for replay in range(4):
        x.copy_(torch.randn(n, channels, generator=g, device="cuda"))
        for t in outs:
            t.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        forth(None), back(None)
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), replay
