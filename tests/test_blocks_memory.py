"""Outputs of norm, the recurrence, the loss and their ways back over other tensors: refused where results would be wrong, and the same bits where
they may lie there."""
import pytest
import torch

from paper_1912_09268_amd import layers_binding as B
from paper_1912_09268_amd import layers

K = 1 << 20                       # addresses K apart, each of a buffer of less; no refused call looks at them
FLOATS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _refused(fn, good, **bad):
    with pytest.raises(B.MgwfbpError) as e:
        fn(*{**good, **bad}.values())
    assert e.value.status == -1, bad


NORM = dict(d_x=K, x_stride=20, dtype=B.BF16, d_residual=2 * K, residual_stride=20, stream_dtype=B.F32, n_tokens=300, n_channels=20, d_weight=3 * K, weight_dtype=B.F32,
            eps=1e-6, d_h=4 * K, h_stride=20, d_y=5 * K, y_stride=20, d_rstd=6 * K, d_q=7 * K, d_scale=8 * K, d_linear_scale=9 * K, ld=32)


@pytest.mark.parametrize("bad", [
    dict(d_y=4 * K), dict(d_y=4 * K + 160), dict(d_h=5 * K - 80, d_y=5 * K),                # outputs over each other
    dict(d_h=K), dict(d_y=2 * K), dict(d_y=K + 40),                                         # over an input of another type, or some rows behind it
    dict(d_h=2 * K, h_stride=21), dict(d_h=2 * K + 80), dict(d_y=K, y_stride=24),
    dict(d_residual=0, d_h=0, stream_dtype=B.BF16, residual_stride=0, h_stride=0, d_y=K),   # y over an x of which n is kept
    dict(d_rstd=3 * K), dict(d_rstd=5 * K + 400), dict(d_q=2 * K), dict(d_q=8 * K), dict(d_linear_scale=8 * K), dict(d_scale=3 * K), dict(d_y=3 * K),
])
def test_norm_refuses(bad):
    _refused(B.norm, NORM, **bad)


NORM_BACK = dict(d_q=K, d_scale=2 * K, ld=32, d_rstd=3 * K, n_tokens=300, n_channels=20, d_weight=4 * K, weight_dtype=B.BF16, d_dy=5 * K, dy_stride=20, dtype=B.BF16,
                 d_dresidual=6 * K, dresidual_stride=20, d_dh=7 * K, dh_stride=20, stream_dtype=B.F32, d_dx=8 * K, dx_stride=20, accumulate=False, d_dw=9 * K,
                 grad_dtype=B.F32, d_workspace=10 * K, workspace_bytes=K)


@pytest.mark.parametrize("bad", [
    dict(d_dx=7 * K), dict(d_dx=7 * K + 40), dict(stream_dtype=B.BF16, d_dx=7 * K),         # dx over dh
    dict(d_dh=5 * K), dict(d_dx=6 * K), dict(d_dh=6 * K, dh_stride=22), dict(d_dh=6 * K + 80), dict(d_dx=5 * K - 40),
    dict(d_dw=4 * K), dict(d_dw=7 * K + 4), dict(d_dh=K), dict(d_dx=2 * K), dict(d_dx=3 * K), dict(d_workspace=7 * K), dict(d_workspace=5 * K), dict(d_dw=10 * K + 64),
])
def test_norm_backward_refuses(bad):
    _refused(B.norm_backward, NORM_BACK, **bad)


ONE, PACKED = B.Sequences(3, 3000, 0, 0), B.Sequences(3, 3000, 20 * K, B.I64)
RECUR = dict(sequences=ONE, n_channels=20, kind=B.UNIT, dtype=B.BF16, d_gate=K, gate_stride=20, d_x=2 * K, x_stride=20, d_first=3 * K, d_y=4 * K, y_stride=20, d_last=5 * K,
             d_states=6 * K, d_workspace=7 * K, workspace_bytes=K)


@pytest.mark.parametrize("bad", [
    dict(d_y=K + 40), dict(d_y=K, y_stride=40), dict(d_y=2 * K, y_stride=21), dict(d_y=2 * K - 40), dict(d_last=3 * K + 80), dict(d_last=3 * K - 80),
    dict(sequences=PACKED, d_last=3 * K), dict(d_states=3 * K), dict(d_states=K), dict(d_last=K), dict(d_states=5 * K), dict(d_y=3 * K), dict(d_workspace=K),
    dict(d_workspace=4 * K), dict(sequences=PACKED, d_states=20 * K), dict(sequences=PACKED, d_last=20 * K + 8), dict(d_y=5 * K - 2),
])
def test_recur_refuses(bad):
    _refused(B.recur, RECUR, **bad)


RECUR_BACK = dict(sequences=ONE, n_channels=20, kind=B.UNIT, dtype=B.BF16, d_gate=K, gate_stride=20, d_x=2 * K, x_stride=20, d_first=3 * K, d_states=4 * K, d_dy=5 * K,
                  dy_stride=20, d_dlast=6 * K, d_dgate=7 * K, dgate_stride=20, d_dx=8 * K, dx_stride=20, d_dfirst=9 * K, d_workspace=10 * K, workspace_bytes=K)


@pytest.mark.parametrize("bad", [
    dict(d_dx=7 * K), dict(d_dx=7 * K + 40), dict(d_dgate=8 * K, dgate_stride=40), dict(d_dx=7 * K + 20, dgate_stride=40, dx_stride=40),       # dgate over dx, in part
    dict(d_dgate=K + 40), dict(d_dx=2 * K, dx_stride=24), dict(d_dx=5 * K - 40), dict(d_dfirst=6 * K), dict(d_dfirst=6 * K + 80), dict(d_dfirst=3 * K), dict(d_dfirst=7 * K),
    dict(d_dgate=4 * K), dict(d_dx=3 * K), dict(d_workspace=8 * K), dict(d_workspace=4 * K), dict(sequences=PACKED, d_dfirst=20 * K),
])
def test_recur_backward_refuses(bad):
    _refused(B.recur_backward, RECUR_BACK, **bad)


LOSS = dict(d_z=K, z_stride=50, dtype=B.F16, n_tokens=90, n_vocabulary=50, d_labels=2 * K, label_type=B.I64, d_ids=3 * K, ids_stride=4, id_type=B.I32, d_teacher=4 * K,
            teacher_stride=4, teacher_dtype=B.BF16, n_top=4, temperature=2.0, label_weight=1.0, teacher_weight=1.0, d_row_weight=5 * K, d_loss=6 * K, d_dz=7 * K, dz_stride=50,
            d_workspace=0, workspace_bytes=0)


@pytest.mark.parametrize("bad", [
    dict(d_loss=5 * K), dict(d_loss=5 * K + 4), dict(d_loss=5 * K - 356), dict(d_loss=7 * K), dict(d_loss=K), dict(d_loss=2 * K), dict(d_loss=3 * K), dict(d_loss=4 * K),
    dict(d_dz=K + 100), dict(d_dz=K, dz_stride=51), dict(d_dz=4 * K), dict(d_dz=5 * K), dict(d_dz=K - 2),
    dict(n_tokens=2, n_vocabulary=40000, z_stride=40000, dz_stride=40000, d_workspace=K + 256, workspace_bytes=K),
])
def test_distill_refuses(bad):
    _refused(B.distill, LOSS, **bad)


@pytest.fixture(params=["native", "plain"])
def way(request, monkeypatch):
    if request.param == "plain":
        for name in ("norm", "norm_backward", "recur", "recur_backward", "distill"):
            monkeypatch.setattr(layers._native, name, lambda *a: NotImplemented)
    return request.param


@pytest.mark.gpu
def test_both_ways_say_what_lies_over_what(way):
    d = "cuda"
    t, c = 300, 48
    x, r, w = torch.randn(t, c, device=d), torch.randn(t, c, device=d), torch.ones(c, device=d)
    low, arena = x.to(torch.bfloat16), torch.zeros(2 * t, c, device=d)
    kept = layers.norm_empty(t, c)
    y, h, dw = torch.zeros(t, c, device=d), torch.zeros(t, c, device=d), torch.zeros(c, device=d)
    layers.norm(x, w, y=y, kept=kept)
    as_low = arena[:t].view(torch.bfloat16)[:, :c]                          # the same memory, another type: every second piece of 2 c bytes
    for says, call in (("h is written and shares memory with residual", lambda: layers.norm(x, w, residual=arena[:t], y=y, h=arena[1:t + 1])),
                       ("h and y", lambda: layers.norm(x, w, residual=r, y=arena[1:t + 1], h=arena[:t])),
                       ("y .* x", lambda: layers.norm(arena[:t], w, y=arena[1:t + 1]))):
        print("[memory]", way, says, flush=True)
        with pytest.raises(ValueError, match=says):
            call()
    with pytest.raises(ValueError, match="dh and dx"):
        layers.norm_backward(kept, low, w, dh=arena[:t], dx=as_low, dw=dw)
    with pytest.raises(ValueError, match="dh .* dy"):
        layers.norm_backward(kept, as_low, w, dh=arena[:t])
    with pytest.raises(ValueError, match="dw .* weight"):
        layers.norm_backward(kept, x, arena.view(-1)[:c], dh=h, dw=arena.view(-1)[1:c + 1])
    states = layers.recur_empty(x)
    layers.recur(x, r, states=states)
    with pytest.raises(ValueError, match="y .* gate"):
        layers.recur(arena[:t], x, y=arena[1:t + 1])
    with pytest.raises(ValueError, match="dgate and dx"):
        layers.recur_backward(x, r, states, y, dgate=h, dx=h)
    with pytest.raises(ValueError, match="dfirst"):
        layers.recur_backward(x, r, states, y, dgate=h, dx=y, dlast=arena[:1], dfirst=arena[:1])
    many = torch.zeros(t + 1, device=d)
    for loss in (many[:t], many[1:]):
        with pytest.raises(ValueError, match="loss .* row_weight"):
            layers.distill(x, labels=torch.zeros(t, dtype=torch.int64, device=d), row_weight=many[:t], loss=loss)
    torch.cuda.synchronize()
    assert not bool(arena.any()) and not bool(h.any()) and not bool(many.any())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("tokens,channels", [(1, 64), (300, 130), (700, 2050), (40, 9000), (20, 20000)])
def test_norm_in_place(tokens, channels, dtype, way):
    print("[memory] norm", tokens, channels, dtype, flush=True)
    T = FLOATS[dtype]
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, r, dy, dres = (torch.randn(tokens, channels, generator=g, device="cuda").to(T) for _ in range(4))
    w = torch.randn(channels, generator=g, device="cuda")
    kept, again = layers.norm_empty(tokens, channels), layers.norm_empty(tokens, channels)
    y, h = layers.norm(x, w, residual=r, kept=kept)
    for over_y, over_h in (("x", "r"), ("r", "x"), (None, "x"), ("x", None), ("r", None)):
        at = {"x": x.clone(), "r": r.clone()}
        y2, h2 = at.get(over_y, torch.empty_like(x)), at.get(over_h, torch.empty_like(x))
        layers.norm(at["x"], w, residual=at["r"], y=y2, h=h2, kept=again)
        assert torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(again.rstd, kept.rstd) and torch.equal(again.act.q[:, :channels], kept.act.q[:, :channels])
    plain = layers.norm(x, w)[0]
    over = x.clone()
    layers.norm(over, w, y=over)
    assert torch.equal(over, plain)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    dh = layers.norm_backward(kept, dy, w, dres=dres, dx=dx, dw=dw)
    for over_h, over_x in (("dy", "dres"), ("dres", "dy"), ("dy", None), (None, "dres")):
        at = {"dy": dy.clone(), "dres": dres.clone()}
        dh2, dx2, dw2 = at.get(over_h, torch.empty_like(x)), at.get(over_x, torch.empty_like(x)), torch.empty_like(w)
        layers.norm_backward(kept, at["dy"], w, dres=at["dres"], dh=dh2, dx=dx2, dw=dw2)
        assert torch.equal(dh2, dh) and torch.equal(dx2, dx) and torch.equal(dw2, dw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("shape,offsets", [((9, 1, 130), None), ((5, 7, 33), None), ((40, 20, 65), None), ((3, 300, 70), None), ((2, 5000, 16), None),
                                           ((700, 40), [0, 3, 3, 200, 690]), ((9000, 20), [0, 4000, 4001, 9000])])
def test_recur_in_place(shape, offsets, dtype, way):
    print("[memory] recur", shape, offsets, dtype, flush=True)
    T = FLOATS[dtype]
    g = torch.Generator(device="cuda").manual_seed(shape[0])
    gate, x, dy = (torch.randn(shape, generator=g, device="cuda").to(T) for _ in range(3))
    offsets = None if offsets is None else torch.tensor(offsets, device="cuda")
    inside = slice(None) if offsets is None else slice(0, int(offsets[-1]))
    states, more = layers.recur_empty(gate, offsets), layers.recur_empty(gate, offsets)
    y = layers.recur(gate, x, kind="unit", offsets=offsets, states=states)
    dgate, dx = layers.recur_backward(gate, x, states, dy, kind="unit", offsets=offsets)
    for over in range(2):
        at = [gate.clone(), x.clone()]
        behind = at[over].clone()
        layers.recur(*at, kind="unit", offsets=offsets, y=at[over], states=more)
        assert torch.equal(at[over][inside], y[inside]) and torch.equal(more, states)
        assert offsets is None or torch.equal(at[over][int(offsets[-1]):], behind[int(offsets[-1]):])
    for i, j in ((0, 1), (1, 0), (0, 2), (2, 0), (1, 2), (2, 1)):
        at = [gate.clone(), x.clone(), dy.clone()]
        layers.recur_backward(at[0], at[1], states, at[2], kind="unit", offsets=offsets, dgate=at[i], dx=at[j])
        assert torch.equal(at[i][inside], dgate[inside]) and torch.equal(at[j][inside], dx[inside]), (i, j)
