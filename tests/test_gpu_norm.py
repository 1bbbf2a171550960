"""Root-mean-square norm with the residual's addition and its 8-bit checkpoint, and the way back, against plain 64-bit implementations.

Tolerances: y is rstd (one rounding) times h times weight, one rounding each, and the rounding of its type.  Codes and steps are compared bit for
bit with their definition from the kernel's own rstd, and rstd with its definition to the last bit of binary32."""
import math

import numpy as np
import pytest
import torch

from paper_1912_09268_amd import layers_binding as M
from paper_1912_09268_amd import layers
from test_gpu_layers import BF16, DT, F16, F32, G, _close, _codes, _gen, _strided, _untouched

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")]
SIZES = [(1, 1024), (1, 1), (3, 7), (5, 128), (130, 129), (67, 512), (257, 520), (128, 1024), (300, 1001), (129, 2048), (40, 2050), (17, 4096), (33, 8192),
         (9, 8200), (5, 16384), (4, 16385), (130, 20001)]


def _say(*a):
    print("[norm]", *a, flush=True)


def _inputs(tokens, channels, dtype, stream, how, seed):
    g = _gen(seed)
    x, _ = _strided((tokens, channels), DT[dtype], how)
    x.copy_(torch.randn(tokens, channels, generator=g, device="cuda") * torch.exp(torch.randn(channels, generator=g, device="cuda")))
    r, _ = _strided((tokens, channels), DT[stream], how)
    r.copy_(torch.randn(tokens, channels, generator=g, device="cuda"))
    w = 1.0 + 0.3 * torch.randn(channels, generator=g, device="cuda")
    return g, x, r, w


def _check_kept(kept, h, rstd64, weight, channels):
    rstd = kept.rstd.double()
    assert bool(((rstd - rstd64).abs() <= 1.001 * U * rstd64).all())
    n = h.float() * kept.rstd[:, None]
    q, scale = _codes(n)
    own = -(-channels // 16) * 16
    assert np.array_equal(kept.act.q[:, :channels].cpu().numpy(), q)
    assert np.array_equal(kept.act.scale[:, :channels].cpu().numpy().view(np.uint32) & 0x7fffffff, scale.view(np.uint32) & 0x7fffffff)
    linear = torch.from_numpy(scale).cuda() * (weight.float() if weight is not None else 1.0)
    assert torch.equal(kept.linear.scale[:, :channels].nan_to_num(nan=-1.0), linear.nan_to_num(nan=-1.0))
    for pad in (kept.act.q[:, channels:own], kept.act.scale[:, channels:own], kept.linear.scale[:, channels:own]):
        assert not bool(pad.any())


@pytest.mark.parametrize("how", ["dense", "strided"])
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("tokens,channels", SIZES)
def test_norm(tokens, channels, dtype, stream, how):
    _say("forward", tokens, channels, dtype, stream, how)
    g, x, r, w = _inputs(tokens, channels, dtype, stream, how, tokens + channels)
    w = w.to(DT[dtype]) if tokens % 2 else w
    eps = 1e-5
    y, y_whole = _strided((tokens, channels), DT[dtype], how)
    h, h_whole = _strided((tokens, channels), DT[stream], how)
    kept = layers.norm_empty(tokens, channels)
    got = layers.norm(x, w, residual=r, y=y, h=h, kept=kept, eps=eps)
    assert got[0] is y and got[1] is h
    want_h = (x.float() + r.float()).to(DT[stream])
    torch.cuda.synchronize()
    assert torch.equal(h, want_h)
    rstd = 1.0 / torch.sqrt(want_h.double().square().mean(1) + eps)
    want = want_h.double() * rstd[:, None] * w.double()
    _close(y, want, 4 * U * want.abs(), "y")
    assert _untouched(y, y_whole, math.nan) and _untouched(h, h_whole, math.nan)
    _check_kept(kept, want_h, rstd, w, channels)
    # nothing kept, no weight; h over the residual: the same bits
    again = torch.empty(tokens, channels, dtype=DT[dtype], device="cuda")
    over = r.clone()
    layers.norm(x, w, residual=over, y=again, h=over, eps=eps)
    assert torch.equal(again, y) and torch.equal(over, h)
    # without a residual
    alone = layers.norm_empty(tokens, channels)
    y2, h2 = layers.norm(x, None, kept=alone, eps=eps)
    assert h2 is x
    rstd = 1.0 / torch.sqrt(x.double().square().mean(1) + eps)
    want = x.double() * rstd[:, None]
    _close(y2, want, 4 * U * want.abs(), "y alone")
    _check_kept(alone, x, rstd, None, channels)


def _back_reference(kept, dy, w, dres):
    """(dh, slack of dh, dw, slack of dw)"""
    tokens, channels = kept.act.q.shape[0], kept.act.channels
    group = torch.arange(tokens, device="cuda") // G
    n = kept.act.q[:, :channels].double() * kept.act.scale.double()[group, :channels]
    d, rstd = dy.double(), kept.rstd.double()[:, None]
    g = d * (1.0 if w is None else w.double())
    mean, terms = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dh = rstd * (g - n * mean)
    # g has one rounding, n one; the mean those of its terms and of a sum of that many, and one of 1/channels
    off = rstd * (4 * U * (g.abs() + (n * mean).abs()) + n.abs() * (channels + 8) * U * terms)
    if dres is not None:
        dh, off = dh + dres.double(), off + U * (dres.double().abs() + dh.abs())
    return dh, off, (d * n).sum(0), (tokens + 8) * U * (d * n).abs().sum(0)


@pytest.mark.parametrize("how", ["dense", "strided"])
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("tokens,channels", SIZES + [(2500, 64), (5000, 1024), (1500, 4104)])
def test_norm_backward(tokens, channels, dtype, stream, how):
    _say("backward", tokens, channels, dtype, stream, how)
    g, x, r, w = _inputs(tokens, channels, dtype, stream, how, tokens * 3 + channels)
    kept = layers.norm_empty(tokens, channels)
    layers.norm(x, w, residual=r, kept=kept)
    dy, _ = _strided((tokens, channels), DT[dtype], how)
    dy.copy_(torch.randn(tokens, channels, generator=g, device="cuda"))
    dres, _ = _strided((tokens, channels), DT[stream], how)
    dres.copy_(torch.randn(tokens, channels, generator=g, device="cuda"))
    dh, whole = _strided((tokens, channels), DT[stream], how)
    dx = torch.empty(tokens, channels, dtype=DT[dtype], device="cuda")
    dw = torch.empty(channels, dtype=DT[stream], device="cuda")
    assert layers.norm_backward(kept, dy, w, dres=dres, dh=dh, dx=dx, dw=dw) is dh
    want, off, want_w, off_w = _back_reference(kept, dy, w, dres)
    _close(dh, want, off, "dh")
    _close(dx, want, off, "dx")
    _close(dw, want_w, off_w, "dw")
    assert _untouched(dh, whole, math.nan)
    # in place, added to what is there: the same bits, the sum
    over, had = dres.clone(), torch.randn(channels, generator=g, device="cuda").to(DT[stream])
    more = had.clone()
    layers.norm_backward(kept, dy, w, dres=over, dh=over, dw=more, accumulate=True)
    assert torch.equal(over, dh)
    _close(more, want_w + had.double(), off_w + 2 * U * had.double().abs(), "dw added")
    # without residual, weight, dw
    alone = layers.norm_backward(kept, dy)
    want, off, _, _ = _back_reference(kept, dy, None, None)
    assert alone.dtype == DT[dtype]
    _close(alone, want, off, "dh alone")


def test_gradients_against_differences():
    """The slope of sum(c * y) along a direction, by differences of the plain 64-bit norm, against what the 8 bits give: codes are off by half a
    step of 1/127 of a channel's largest, so the products with n^ by 1/254 of that."""
    g = _gen(8)
    tokens, channels = 64, 96
    x = torch.randn(tokens, channels, generator=g, device="cuda")
    w = 1 + 0.2 * torch.randn(channels, generator=g, device="cuda")
    c = torch.randn(tokens, channels, generator=g, device="cuda")
    kept = layers.norm_empty(tokens, channels)
    layers.norm(x, w, kept=kept)
    dw = torch.empty(channels, device="cuda")
    dh = layers.norm_backward(kept, c, w, dw=dw).double()

    def loss(x, w):
        return float((x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * w * c.double()).sum())

    for seed in range(4):
        v = torch.randn(tokens, channels, generator=_gen(100 + seed), device="cuda").double()
        u = torch.randn(channels, generator=_gen(200 + seed), device="cuda").double()
        e = 1e-5
        along = (loss(x.double() + e * v, w.double()) - loss(x.double() - e * v, w.double())) / (2 * e)
        along_w = (loss(x.double(), w.double() + e * u) - loss(x.double(), w.double() - e * u)) / (2 * e)
        # n^ is off by at most half a step each; in dh it stands twice beside the mean of |g|, in dw once beside dy
        step = (kept.act.scale[:1, :channels].double() / 2)
        n = x.double() * kept.rstd.double()[:, None]
        gw = (c * w).double().abs()
        bound = (kept.rstd.double()[:, None] * (step * (gw * n.abs()).mean(1, keepdim=True) + (n.abs() + step) * (gw * step).mean(1, keepdim=True)) * v.abs()).sum()
        assert abs(along - float((dh * v).sum())) <= float(bound) + 1e-4
        assert abs(along_w - float((dw.double() * u).sum())) <= float((c.double().abs() * step * u.abs()).sum()) + 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_that_are_zero_enormous_or_not_finite(dtype):
    _say("odd rows", dtype)
    tokens, channels = 300, 200
    x = torch.randn(tokens, channels, generator=_gen(1), device="cuda").to(DT[dtype])
    x[0] = 0.0
    x[1] = 6e4 if dtype == "f16" else 3e38
    x[2] = 6e-8 if dtype == "f16" else 1e-38
    x[200, 5] = math.inf
    x[201, 6] = math.nan
    kept = layers.norm_empty(tokens, channels)
    y, _ = layers.norm(x, kept=kept)
    torch.cuda.synchronize()
    assert bool((y[0] == 0).all()) and bool(((y[1].double() - 1).abs() < 2.0 ** -7).all())
    assert bool(y[200:202].isnan().any(1).all()) and bool(y[:200].isfinite().all()) and bool(y[202:].isfinite().all())
    # infinity by rstd = 0: NaN at its place, 0 elsewhere; the NaN takes its whole row, so every channel of the group
    assert bool(kept.act.scale[1, :channels].isnan().all()) and not bool(kept.act.q[128:256].any())
    assert bool(kept.act.scale[0, :channels].isfinite().all()) and bool(kept.act.scale[2, :channels].isfinite().all())
    dw = torch.empty(channels, device="cuda")
    dh = layers.norm_backward(kept, torch.ones_like(x), dw=dw)
    assert bool(dh[128:256].isnan().all()) and bool(dw.isnan().all())
    assert bool(dh[:1].isfinite().all()) and bool(dh[256:].isfinite().all())


def test_the_linear_layer_behind_reads_the_same_codes():
    """kept.linear is a checkpoint of n * weight: act_linear_grad from it against y's own."""
    g = _gen(6)
    tokens, channels, outputs = 700, 264, 40
    x = torch.randn(tokens, channels, generator=g, device="cuda").to(BF16)
    w = 1.0 + 0.5 * torch.randn(channels, generator=g, device="cuda")
    w[3], w[4] = 0.0, -2.0
    kept = layers.norm_empty(tokens, channels)
    layers.norm(x, w, kept=kept)
    dy = torch.randn(tokens, outputs, generator=g, device="cuda").to(BF16)
    dw, db = torch.empty(outputs, channels, device="cuda"), torch.empty(outputs, device="cuda")
    layers.act_linear_grad(dy, kept.linear, dw, db=db)
    n = kept.act.q[:, :channels].double() * kept.act.scale.double().repeat_interleave(G, 0)[:tokens, :channels]
    x64, d64 = n * w.double(), dy.double()
    want, terms = (d64.t() @ x64), d64.abs().t() @ x64.abs()
    _close(dw, want, (tokens + 8) * U * terms, "dw")
    assert bool((dw[:, 3] == 0).all())


def test_sizes_of_zero_and_offsets_beyond_32_bits():
    for tokens, channels in ((0, 8), (8, 0), (0, 0)):
        kept = layers.norm_empty(tokens, channels)
        y, _ = layers.norm(torch.empty(tokens, channels, device="cuda"), kept=kept)
        dw = torch.ones(channels, device="cuda")
        assert layers.norm_backward(kept, y, dw=dw).shape == (tokens, channels)
        assert bool((dw == 0).all())
        dw = torch.ones(channels, device="cuda")
        layers.norm_backward(kept, y, dw=dw, accumulate=True)
        assert bool((dw == 1).all())
    rows, stride, channels = 530000, 8192, 40
    _say("offsets beyond 2^32 elements")
    memory = torch.zeros(rows * stride, dtype=BF16, device="cuda")
    x = torch.as_strided(memory, (rows, channels), (stride, 1))
    x[-200:] = torch.randn(200, channels, generator=_gen(2), device="cuda").to(BF16)
    kept = layers.norm_empty(rows, channels)
    y = torch.empty(rows, channels, dtype=BF16, device="cuda")
    layers.norm(x, y=y, kept=kept)
    small = layers.norm(x[-200:].contiguous())[0]
    assert torch.equal(y[-200:], small) and not bool(y[:-200].any())
    dh = layers.norm_backward(kept, y, dres=y, dh=x)                     # written far out, too
    want, off, _, _ = _back_reference(layers.Norm8(layers.Act8(kept.act.q[-256:], kept.act.scale[-3:], channels), kept.rstd[-256:], kept.linear), y[-256:], None, y[-256:]) \
        if rows % G == 0 else (None,) * 4
    at = torch.arange(rows - 200, rows, device="cuda")
    n = kept.act.q[at][:, :channels].double() * kept.act.scale.double()[at // G][:, :channels]
    d = y[at].double()
    want = d + kept.rstd.double()[at, None] * (d - n * (d * n).mean(1, keepdim=True))
    _close(dh[-200:], want, 64 * U * (1 + want.abs()) * (1 + kept.rstd.double()[at, None]) * (1 + n.abs()), "dh far out")


def test_captured_beside_eager_calls():
    """A graph of norm and its way back, replayed with the program's own work between the replays."""
    g = _gen(12)
    tokens, channels = 300, 520
    x, r = torch.randn(tokens, channels, generator=g, device="cuda").to(BF16), torch.randn(tokens, channels, generator=g, device="cuda")
    w, dy = torch.randn(channels, generator=g, device="cuda"), torch.randn(tokens, channels, generator=g, device="cuda").to(BF16)
    kept, y, h, dh, dw = layers.norm_empty(tokens, channels), torch.empty_like(x), torch.empty_like(r), torch.empty_like(r), torch.empty(channels, device="cuda")

    def step():
        layers.norm(x, w, residual=r, y=y, h=h, kept=kept)
        layers.norm_backward(kept, dy, w, dres=r, dh=dh, dw=dw)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for replay in range(4):
        x.copy_(torch.randn(tokens, channels, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, h, dh, dw, kept.act.q, kept.act.scale, kept.rstd)]
        for t in (y, h, dh, dw, kept.act.q, kept.act.scale, kept.rstd):
            t.zero_()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, h, dh, dw, kept.act.q, kept.act.scale, kept.rstd))), replay
