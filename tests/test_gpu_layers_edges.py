"""The gradient operators at the ends of their ranges: values that are not finite or enormous, checkpoints in larger memory, tensors
that autograd follows, and the forms that only long calls take.  References and tolerances as in test_gpu_layers.py."""
import math

import numpy as np
import pytest
import torch

from paper_1912_09268_amd import layers_binding as M
from paper_1912_09268_amd import layers
from test_gpu_layers import BF16, DT, F16, F32, G, OWN, _checkpoint, _close, _embed_grad_reference, _f64, _gen, _linear_slack, _say, _spread, _strided, _untouched

pytestmark = pytest.mark.gpu

KINDS = ["identity", "gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", KINDS)
def test_values_of_f_at_the_ends_of_the_range(kind, dtype):
    """f(x) where x is infinite, NaN or as large as the type holds: f(inf) = inf; f(-inf) is -inf * 0 = NaN (identity: -inf)."""
    _say("f at the ends", kind, dtype)
    ends = [math.inf, -math.inf, math.nan, 3e38, -3e38, 1e25, -1e25, 5e19, -5e19, 65504.0, -65504.0, 100.0, -100.0, 0.0, 1.0, -1.0]
    x = torch.tensor(ends, device="cuda").to(DT[dtype]).repeat(130, 1)
    y = torch.empty_like(x)
    layers.act_store(x, kind=kind, y=y)
    x64 = x.double()
    finite = x64.isfinite()
    want, _ = _f64(kind, torch.where(finite, x64, 0.0))
    below = -math.inf if kind == "identity" else math.nan
    want = torch.where(finite, want, torch.where(x64 == math.inf, math.inf, torch.where(x64 == -math.inf, below, math.nan)))
    # beyond 64 the functions are x or 0 to all digits
    _close(y, want, OWN * x64.abs().nan_to_num(nan=0.0).clamp(max=64.0), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", KINDS)
def test_slopes_of_enormous_activations(kind, dtype):
    """The slope is 1 above and 0 below, however large a finite x^ is; y is x^ or 0."""
    _say("slopes far out", kind, dtype)
    size = torch.tensor([3e38, 1e30, 1e25, 5e19, 1e19, 1e13, 1e6, 1000.0, 100.0, 65.0, 64.0, 63.0, 20.0, 1.0, 0.0, 0.5], device="cuda")
    act = layers.act_empty(130, 16)
    act.q.copy_(torch.tensor([127, -127, 1, -1, 0, 63, -64], device="cuda").repeat(19)[:130, None].expand(130, 16))
    act.scale.copy_((size / 127).expand(2, 16))
    held = act.q.float() * act.scale.repeat_interleave(G, 0)[:130]
    assert bool(held.isfinite().all())
    dy = torch.randn(130, 16, generator=_gen(4), device="cuda").to(DT[dtype])
    value, slope = _f64(kind, held.double())
    y = torch.empty_like(dy) if dtype != "f16" else None                  # binary16 does not hold such a y
    dx = layers.act_backward(act, dy, kind=kind, y=y)
    _close(dx, dy.double() * slope, OWN * dy.double().abs(), "dx")
    if y is not None:
        _close(y, value, OWN * held.double().abs().clamp(max=64.0), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,channels,ld", [(1, 1, 32), (130, 16, 64), (200, 17, 48), (129, 120, 256), (300, 130, 304), (5, 128, 1024)])
def test_act_store_leaves_columns_behind_its_own(tokens, channels, ld, dtype):
    """Zeros from the last channel to the next multiple of 16, nothing behind it."""
    _say("act_store in a wider checkpoint", tokens, channels, ld, dtype)
    x = torch.randn(tokens, channels, generator=_gen(tokens), device="cuda").to(DT[dtype])
    own = -(-channels // 16) * 16
    act = layers.Act8(torch.full((tokens, ld), 77, dtype=torch.int8, device="cuda"), torch.full((-(-tokens // G), ld), 5.0, device="cuda"), channels)
    layers.act_store(x, act, kind="silu", y=torch.empty_like(x))
    alone = layers.act_store(x)
    assert torch.equal(act.q[:, :own], alone.q) and torch.equal(act.scale[:, :own], alone.scale)
    assert not bool(act.q[:, channels:own].any()) and not bool(act.scale[:, channels:own].any())
    assert bool((act.q[:, own:] == 77).all()) and bool((act.scale[:, own:] == 5.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,outputs", [(1, 8), (100, 40), (129, 33), (2000, 64), (5000, 24)])
def test_checkpoints_side_by_side(tokens, outputs, dtype):
    """Several checkpoints in the columns of one memory, each made, gone back through and summed by itself: as those alone."""
    _say("checkpoints side by side", tokens, outputs, dtype)
    widths = [20, 16, 100, 1, 48]
    ld = sum(-(-w // 16) * 16 for w in widths)
    groups, g, code = -(-tokens // G), _gen(tokens), {"f32": M.F32, "bf16": M.BF16, "f16": M.F16}[dtype]
    q, scale = torch.full((tokens, ld), 77, dtype=torch.int8, device="cuda"), torch.full((groups, ld), math.nan, device="cuda")
    parts, at = [], 0
    for w in widths:
        x = torch.randn(tokens, w, generator=g, device="cuda").to(DT[dtype])
        M.act_store(x.data_ptr(), w, code, tokens, w, M.GELU, q.data_ptr() + at, scale.data_ptr() + 4 * at, ld, 0, 0)
        parts.append((at, w, x))
        at += -(-w // 16) * 16
    dy = torch.randn(tokens, outputs, generator=g, device="cuda").to(DT[dtype])
    space = torch.empty(max(M.act_linear_grad_workspace(tokens, max(widths), outputs), M.act_linear_grad_workspace(tokens, 1, outputs)) + 256, dtype=torch.uint8, device="cuda")
    for at, w, x in parts:
        alone, own = layers.act_store(x), -(-w // 16) * 16
        assert torch.equal(q[:, at:at + own], alone.q) and torch.equal(scale[:, at:at + own], alone.scale)
        up, dx, y = torch.randn(tokens, w, generator=g, device="cuda").to(DT[dtype]), torch.empty_like(x), torch.empty_like(x)
        M.act_backward(q.data_ptr() + at, scale.data_ptr() + 4 * at, ld, tokens, w, M.GELU, up.data_ptr(), w, dx.data_ptr(), w, y.data_ptr(), w, code)
        y_alone = torch.empty_like(x)
        assert torch.equal(dx, layers.act_backward(alone, up, kind="gelu", y=y_alone)) and torch.equal(y, y_alone)
        dw, db = torch.empty(outputs, w, device="cuda"), torch.empty(outputs, device="cuda")
        M.act_linear_grad(q.data_ptr() + at, scale.data_ptr() + 4 * at, ld, tokens, w, dy.data_ptr(), outputs, code, outputs, False, dw.data_ptr(), w, db.data_ptr(), M.F32,
                          space.data_ptr(), space.numel())
        dw_alone, db_alone = torch.empty_like(dw), torch.empty_like(db)
        layers.act_linear_grad(dy, alone, dw_alone, db=db_alone)
        assert torch.equal(dw, dw_alone) and torch.equal(db, db_alone)


def _calls():
    """Each operator on plain tensors: (name, tensors read, tensors written, call of all of them)."""
    table, ids, x = torch.randn(30, 48, device="cuda"), torch.arange(64, device="cuda") % 30, torch.randn(64, 48, device="cuda")
    act = layers.act_store(x)

    def memory(*shape):
        return torch.zeros(*shape, device="cuda")

    return [("embed", [table], [memory(64, 48)], lambda r, w: layers.embed(r[0], ids, out=w[0])),
            ("embed_grad", [x], [memory(30, 48)], lambda r, w: layers.embed_grad(r[0], ids, w[0])),
            ("act_store", [x], [torch.empty_like(act.q), torch.empty_like(act.scale), memory(64, 48)],
             lambda r, w: layers.act_store(r[0], layers.Act8(w[0], w[1], 48), kind="gelu", y=w[2])),
            ("act_backward", [x], [memory(64, 48), memory(64, 48)], lambda r, w: layers.act_backward(act, r[0], kind="gelu", dx=w[0], y=w[1])),
            ("act_linear_grad", [x], [memory(48, 48), memory(48)], lambda r, w: layers.act_linear_grad(r[0], act, w[0], db=w[1]))]


@pytest.mark.parametrize("way", ["native", "plain"])
def test_written_tensors_are_marked_as_changed(way, monkeypatch):
    """A tensor that autograd has saved and a call has written since is noticed, as after any other change in place."""
    if way == "plain":
        for name in ("embed", "embed_grad", "act_store", "act_backward", "act_linear_grad"):
            monkeypatch.setattr(layers._native, name, lambda *a: NotImplemented)
    for name, read, written, call in _calls():
        _say("versions", way, name)
        before = [t._version for t in written]
        call(read, written)
        assert all(t._version > b for t, b in zip(written, before)), name
        assert all(t._version == 0 for t in read), name
        a = torch.ones_like(written[-1], requires_grad=True)
        loss = (a * written[-1]).sum()                                    # saves what was written
        call(read, written)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():
        kept = [([t.clone() for t in read], [t.clone() for t in written], call) for _, read, written, call in _calls()]
        for read, written, call in kept:
            call(read, written)
    for read, written, call in kept:                                      # tensors that have no version
        call(read, written)


@pytest.mark.parametrize("way", ["native", "plain"])
def test_tensors_that_autograd_follows_are_refused(way, monkeypatch):
    """The operators have no graph: a gradient would be lost without a word.  Without grad mode, and detached, they are taken."""
    if way == "plain":
        for name in ("embed", "embed_grad", "act_store", "act_backward", "act_linear_grad"):
            monkeypatch.setattr(layers._native, name, lambda *a: NotImplemented)
    for name, read, written, call in _calls():
        _say("autograd", way, name)
        call(read, written)
        want = [t.clone() for t in written]
        followed = [t.clone().requires_grad_(True) for t in read]
        with pytest.raises(ValueError, match="autograd"):
            call(followed, written)
        if written[-1].is_floating_point():
            with pytest.raises(ValueError, match="autograd"):
                call(read, written[:-1] + [written[-1].clone().requires_grad_(True)])
        for t in written:
            t.zero_()
        with torch.no_grad():
            call(followed, written)
        assert all(torch.equal(a, b) for a, b in zip(want, written)), name
        call([t.detach() for t in followed], written)
        with pytest.raises(ValueError, match="autograd"):
            call([t * 1.0 for t in followed], written)
    with pytest.raises(ValueError, match="autograd"):
        layers.embed(torch.zeros(3, 4, device="cuda", requires_grad=True), torch.zeros(2, dtype=torch.int64, device="cuda"))


def test_negated_views_are_refused():
    """A tensor whose memory holds the negative of its values (the imaginary part of a conjugate)."""
    x = torch.complex(torch.zeros(64, 1, device="cuda"), torch.ones(64, 1, device="cuda")).conj().imag
    assert x.is_neg() and bool((x == -1.0).all())
    with pytest.raises(ValueError, match="negat"):
        layers.act_store(x)
    with pytest.raises(ValueError, match="negat"):
        layers.act_store(x, layers.act_empty(64, 1))
    ids = torch.arange(64, device="cuda")
    with pytest.raises(ValueError, match="negat"):
        layers.embed(x, ids, out=torch.empty(64, 1, device="cuda"))
    with pytest.raises(ValueError, match="negat"):
        layers.embed(x.resolve_neg(), torch._neg_view(ids), out=torch.empty(64, 1, device="cuda"))
    with pytest.raises(ValueError, match="negat"):
        layers.embed_grad(torch.ones(64, 8, device="cuda"), ids, torch._neg_view(torch.empty(64, 8, device="cuda")))
    assert bool((layers.embed(x.resolve_neg(), ids, dtype=F32) == -1.0).all())


def test_memory_that_cannot_be_had_is_torchs_own_error():
    """For a workspace, as for a tensor: callers that free and try again catch torch.OutOfMemoryError."""
    tokens, rows, dim = 1 << 20, 5, 1                                     # a workspace of some 25 MB
    dy, ids, grad = torch.ones(tokens, dim, device="cuda"), torch.zeros(tokens, dtype=torch.int64, device="cuda"), torch.empty(rows, dim, device="cuda")
    layers.embed_grad(dy[:300], ids[:300], grad)                          # the library is loaded
    assert M.embed_grad_workspace(tokens, rows, dim) > 4 << 20
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(1e-9)
    held, size = [], 1 << 36                                              # what torch still has of earlier tests' memory, taken
    try:
        while size >= 1 << 20:
            try:
                held.append(torch.empty(size, dtype=torch.uint8, device="cuda"))
            except torch.OutOfMemoryError:
                size //= 2
        with pytest.raises(torch.OutOfMemoryError):
            layers.embed_grad(dy, ids, grad)
    finally:
        held.clear()
        torch.cuda.set_per_process_memory_fraction(1.0)
    layers.embed_grad(dy, ids, grad)
    assert float(grad[0, 0]) == tokens and not bool(grad[1:].any())


def test_tensors_that_are_no_matrix_are_refused_with_the_reason():
    """What cannot be seen as [tokens, dim] without a copy, or has another number of elements: ValueError, as for any other shape."""
    table, ids = torch.randn(10, 24, device="cuda"), torch.arange(12, device="cuda").view(3, 4) % 10
    dy, grad = torch.ones(3, 5, 24, device="cuda"), torch.empty(10, 24, device="cuda")
    with pytest.raises(ValueError, match="dy"):
        layers.embed_grad(dy[:, :4], ids, grad)                           # rows of two strides
    with pytest.raises(ValueError, match="dy"):
        layers.embed_grad(dy, ids, grad)                                  # 15 tokens for 12 ids
    with pytest.raises(ValueError, match="dy"):
        layers.embed_grad(dy[0, 0], ids, grad)
    with pytest.raises(ValueError, match="out"):
        layers.embed(table, ids, out=torch.empty(3, 5, 24, device="cuda")[:, :4])
    whole = torch.empty(3, 4, 30, device="cuda")                          # rows of one stride: taken
    assert torch.equal(layers.embed(table, ids, out=whole[..., :24]), table[ids])
    assert torch.equal(layers.embed_grad(torch.ones(3, 4, 30, device="cuda")[..., :24], ids, grad), torch.bincount(ids.view(-1), minlength=10).float()[:, None].expand(-1, 24))


@pytest.mark.parametrize("spread", ["words", "one", "holes"])
@pytest.mark.parametrize("tokens,rows,dim,dy_t,grad_t,how", [(17003, 30522, 1024, F32, F32, "dense"), (33001, 700, 520, BF16, BF16, "strided"),
                                                             (65543, 30522, 1024, F32, F32, "dense"), (70001, 40, 1021, F16, F32, "strided")])
def test_embed_grad_of_long_chunks(tokens, rows, dim, dy_t, grad_t, how, spread):
    """Chunks of 32 tokens (from 2.1 million vectors of eight on) and of 64 (from 8.4 million): several turns within a chunk, stretches that
    go on behind it."""
    _say("embed_grad, long chunks", tokens, rows, dim, dy_t, grad_t, how, spread)
    vectors = tokens * -(-dim // 8)
    assert vectors >= 64 * 131072 or vectors >= 32 * 65536
    g = _gen(tokens)
    ids = _spread(tokens, rows, spread, g).to(torch.int32 if tokens % 3 == 0 else torch.int64)
    dy, _ = _strided((tokens, dim), dy_t, how)
    dy.copy_(torch.randn(tokens, dim, generator=g, device="cuda"))
    dy[(ids < 0) | (ids >= rows)] = float("nan")
    grad, whole = _strided((rows, dim), grad_t, how)
    scale = 0.37
    layers.embed_grad(dy, ids, grad, scale=scale)
    want, terms, count = _embed_grad_reference(dy, ids, rows, float(np.float32(scale)), -1)
    _close(grad, want, (count + 2) * 2.0 ** -24 * terms, "embed_grad")
    assert _untouched(grad, whole, float("nan"))
    again = grad.clone()
    layers.embed_grad(dy, ids, grad, scale=scale)
    assert torch.equal(again, grad)
    had = torch.randn(rows, dim, generator=g, device="cuda").to(grad_t)
    grad.copy_(had)
    pad = int(ids[0])
    layers.embed_grad(dy, ids, grad, scale=scale, padding_row=pad, accumulate=True)
    if 0 <= pad < rows:
        want[pad], terms[pad], count[pad] = 0.0, 0.0, 0.0
    _close(grad, want + had.double(), (count + 3) * 2.0 ** -24 * (terms + had.double().abs()), "accumulated")
    rest = count.squeeze(1) == 0
    assert torch.equal(grad[rest], had[rest])


@pytest.mark.parametrize("dy_t,grad_t", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("tokens,channels,outputs,how", [(32, 16392, 8200, "dense"), (77, 16385, 8203, "strided")])
def test_act_linear_grad_of_gradients_past_the_caches(tokens, channels, outputs, how, dy_t, grad_t):
    """dw of 256 MiB and more by few tokens: streamed tiles, whole and at the edges, and added to what is there."""
    _say("act_linear_grad, streamed", tokens, channels, outputs, how, dy_t, grad_t)
    assert outputs * channels * (4 if grad_t == "f32" else 2) >= 256 << 20
    g = _gen(tokens)
    act, x = _checkpoint(tokens, channels, g)
    dy = torch.randn(tokens, outputs, generator=g, device="cuda").to(DT[dy_t])
    dw, whole = _strided((outputs, channels), DT[grad_t], how)
    db = torch.empty(outputs, dtype=DT[grad_t], device="cuda")
    layers.act_linear_grad(dy, act, dw, db=db)
    had = torch.randn(outputs, channels, generator=g, device="cuda").to(DT[grad_t])
    first = dw.clone()
    assert _untouched(dw, whole, float("nan"))
    dw.copy_(had)
    layers.act_linear_grad(dy, act, dw, accumulate=True)
    d64 = dy.double().t().contiguous()
    _close(db, d64.sum(1), (tokens + 8) * 2.0 ** -24 * d64.abs().sum(1), "db")
    for o in range(0, outputs, 2048):                                     # in parts: the references are 64 bits
        part = slice(o, min(o + 2048, outputs))
        want, terms = d64[part] @ x, d64[part].abs() @ x.abs()
        _close(first[part], want, _linear_slack(tokens, terms, 0.0), "dw")
        h = had[part].double()
        _close(dw[part], want + h, _linear_slack(tokens, terms, h.abs()), "accumulated dw")


@pytest.mark.parametrize("kind", KINDS[1:])
def test_the_tails_keep_their_digits(kind):
    """f(x) far below 0 relative to itself.  The exponential's argument has the roundings of binary32: three of 2^-24 of it each
    for GELU (x^2, the constant, the product) and tanh GELU has the polynomial's two beside them, so f is off by that many parts of
    |argument| beside the function's own error.  Where f is below 2^-100 nothing is asked."""
    x = -torch.linspace(0.5, 14.0, 128 * 64, device="cuda").view(128, 64)
    y = torch.empty_like(x)
    layers.act_store(x, kind=kind, y=y)
    x64 = x.double()
    want, _ = _f64(kind, x64)
    argument = {"gelu": x64 * x64 / 2, "silu": x64.abs(), "gelu_tanh": 2 * math.sqrt(2 / math.pi) * (x64.abs() + 0.044715 * x64.abs() ** 3)}[kind]
    roundings = {"gelu": 3, "silu": 2, "gelu_tanh": 6}[kind]
    slack = (OWN + roundings * 2.0 ** -24 * argument) * want.abs() + 2.0 ** -100
    _close(y, want, slack, "y")
    assert bool((want.abs() > 2.0 ** -90).sum() > 4000)
