"""What norm, the recurrence and the loss refuse: at the C entry points (checked before anything touches a GPU) and on torch tensors."""
import ctypes as C
import math

import pytest
import torch

from paper_1912_09268_amd import layers_binding as B
from paper_1912_09268_amd import layers

P = 1 << 12                       # an aligned address that no refused call looks at


def _refused(fn, *args):
    with pytest.raises(B.MgwfbpError) as e:
        fn(*args)
    assert e.value.status == -1


def test_norm_refuses():
    good = dict(d_x=P, x_stride=20, dtype=B.BF16, d_residual=P, residual_stride=20, stream_dtype=B.F32, n_tokens=9, n_channels=20, d_weight=P, weight_dtype=B.F32,
                eps=1e-6, d_h=P, h_stride=20, d_y=P, y_stride=20, d_rstd=P, d_q=P, d_scale=P, d_linear_scale=P, ld=32)
    for bad in (dict(d_x=0), dict(d_x=P + 1), dict(x_stride=19), dict(dtype=3), dict(dtype=B.F16, stream_dtype=B.BF16), dict(dtype=B.F32, stream_dtype=B.BF16),
                dict(d_residual=0), dict(d_h=0), dict(d_residual=P + 2), dict(residual_stride=19), dict(h_stride=19), dict(d_h=P + 2),
                dict(d_residual=0, d_h=0), dict(n_tokens=-1), dict(n_tokens=2 ** 26 + 1), dict(n_channels=-1), dict(n_channels=2 ** 23 + 1), dict(d_weight=P + 2),
                dict(weight_dtype=7), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(d_y=0), dict(d_y=P + 1), dict(y_stride=19), dict(d_rstd=0),
                dict(d_q=0), dict(d_scale=0), dict(d_linear_scale=0), dict(d_rstd=P + 2), dict(d_q=P + 8), dict(d_scale=P + 4), dict(d_linear_scale=P + 4), dict(ld=16),
                dict(ld=40), dict(d_y=4 * P, d_h=4 * P), dict(d_residual=0, d_h=0, stream_dtype=B.BF16, d_y=P), dict(d_h=P, residual_stride=21), dict(d_residual=2 * P, d_h=2 * P, h_stride=24)):
        _refused(B.norm, *{**good, **bad}.values())
    wide = dict(n_tokens=2 ** 24, n_channels=9000, d_h=2 * P, d_y=4 * P, **{k: 9000 for k in ("x_stride", "residual_stride", "h_stride", "y_stride")}, d_rstd=0, d_q=0,
                d_scale=0, d_linear_scale=0)                          # 2^34 lanes
    _refused(B.norm, *{**good, **wide}.values())
    B.norm(*{**good, "n_tokens": 0, "d_x": 0, "d_residual": 0, "d_y": 0, "d_q": 0}.values())
    back = dict(d_q=P, d_scale=P, ld=32, d_rstd=P, n_tokens=9, n_channels=20, d_weight=P, weight_dtype=B.BF16, d_dy=P, dy_stride=20, dtype=B.BF16, d_dresidual=P,
                dresidual_stride=20, d_dh=P, dh_stride=20, stream_dtype=B.F32, d_dx=P, dx_stride=20, accumulate=False, d_dw=P, grad_dtype=B.F32, d_workspace=P,
                workspace_bytes=1 << 20)
    for bad in (dict(d_q=0), dict(d_q=P + 8), dict(d_scale=0), dict(d_scale=P + 8), dict(ld=20), dict(ld=16), dict(d_rstd=0), dict(n_tokens=-1), dict(n_tokens=2 ** 26 + 1),
                dict(n_channels=2 ** 23 + 1), dict(d_weight=P + 1), dict(weight_dtype=-1), dict(d_dy=0), dict(dy_stride=19), dict(dtype=9), dict(d_dresidual=P + 2),
                dict(dresidual_stride=19), dict(d_dh=0), dict(dh_stride=19), dict(stream_dtype=B.F16), dict(d_dx=P + 1), dict(dx_stride=19), dict(d_dw=P + 2), dict(grad_dtype=3),
                dict(d_dh=P, dh_stride=21), dict(d_workspace=0), dict(d_workspace=P + 64), dict(workspace_bytes=B.norm_backward_workspace(9, 20) - 1),
                dict(n_channels=20000, ld=20000, dy_stride=20000, dh_stride=20000, dx_stride=20000, dresidual_stride=20000, d_dw=0, d_workspace=0)):
        _refused(B.norm_backward, *{**back, **bad}.values())
    B.norm_backward(*{**back, "n_tokens": 0, "d_q": 0, "d_dw": 0, "d_workspace": 0}.values())
    _refused(B.norm_backward_workspace, -1, 1)
    assert B.lib().mgwfbp_norm_backward_workspace(1, 1, None) == -1 and B.norm_backward_workspace(0, 5) == 0


def test_recur_refuses():
    one, packed = B.Sequences(3, 3000, 0, 0), B.Sequences(3, 3000, P, B.I64)
    good = dict(sequences=one, n_channels=20, kind=B.UNIT, dtype=B.BF16, d_gate=P, gate_stride=20, d_x=P, x_stride=20, d_first=P, d_y=P, y_stride=20, d_last=2 * P,
                d_states=P, d_workspace=P, workspace_bytes=1 << 20)
    back = dict(sequences=one, n_channels=20, kind=B.UNIT, dtype=B.BF16, d_gate=P, gate_stride=20, d_x=P, x_stride=20, d_first=P, d_states=P, d_dy=P, dy_stride=20,
                d_dlast=P, d_dgate=P, dgate_stride=20, d_dx=P, dx_stride=20, d_dfirst=2 * P, d_workspace=P, workspace_bytes=1 << 20)
    wrong = [B.Sequences(-1, 300, 0, 0), B.Sequences(7, 300, 0, 0), B.Sequences(3, -3, 0, 0), B.Sequences(3, 3 * 2 ** 25, 0, 0), B.Sequences(0, 5, 0, 0), B.Sequences(3, 300, P + 4, B.I64),
             B.Sequences(3, 300, P, 2), B.Sequences(2 ** 26 + 1, 0, 0, 0)]
    assert B.recur_workspace(one, 20, B.BF16) > 0
    common = [dict(sequences=s) for s in wrong] + [dict(n_channels=-1), dict(n_channels=2 ** 23 + 1), dict(kind=3), dict(kind=-1), dict(dtype=3), dict(d_gate=0), dict(d_gate=P + 1),
                                                   dict(gate_stride=19), dict(d_x=0), dict(x_stride=19), dict(d_first=P + 2), dict(d_states=P + 1), dict(d_workspace=0),
                                                   dict(d_workspace=P + 128), dict(workspace_bytes=B.recur_workspace(one, 20, B.BF16) - 1)]
    for bad in common + [dict(d_y=0), dict(y_stride=19), dict(d_last=P + 2), dict(sequences=packed, d_last=P)]:
        _refused(B.recur, *{**good, **bad}.values())
    for bad in common + [dict(d_states=0), dict(d_dy=0), dict(dy_stride=19), dict(d_dlast=P + 2), dict(d_dgate=0), dict(dgate_stride=19), dict(d_dx=0), dict(dx_stride=19),
                         dict(d_dfirst=P + 1), dict(d_dfirst=P)]:
        _refused(B.recur_backward, *{**back, **bad}.values())
    none = B.Sequences(0, 0, 0, 0)
    B.recur(*{**good, "sequences": none, "d_gate": 0}.values())
    B.recur_backward(*{**back, "sequences": none, "d_gate": 0}.values())
    assert B.lib().mgwfbp_recur_states(C.byref(one), None) == -1 and B.lib().mgwfbp_recur_workspace(None, 1, 0, None) == -1
    assert (B.recur_states(one), B.recur_states(packed), B.recur_states(B.Sequences(2, 258, 0, 0)), B.recur_states(none)) == (24, 24, 4, 0)
    for s in wrong:
        _refused(B.recur_states, s)
        _refused(B.recur_workspace, s, 8, B.F32)


def test_distill_refuses():
    good = dict(d_z=P, z_stride=50, dtype=B.F16, n_tokens=9, n_vocabulary=50, d_labels=P, label_type=B.I64, d_ids=P, ids_stride=4, id_type=B.I32, d_teacher=P, teacher_stride=4,
                teacher_dtype=B.BF16, n_top=4, temperature=2.0, label_weight=1.0, teacher_weight=1.0, d_row_weight=P, d_loss=P, d_dz=P, dz_stride=50,
                d_workspace=0, workspace_bytes=0)
    for bad in (dict(d_z=0), dict(d_z=P + 1), dict(z_stride=49), dict(dtype=3), dict(n_tokens=-1), dict(n_tokens=2 ** 26 + 1), dict(n_vocabulary=0), dict(n_vocabulary=2 ** 23 + 1),
                dict(d_labels=P + 4), dict(label_type=2), dict(d_ids=0), dict(d_ids=P + 2), dict(ids_stride=3), dict(id_type=-1), dict(d_teacher=0), dict(d_teacher=P + 1),
                dict(teacher_stride=3), dict(teacher_dtype=4), dict(n_top=-1), dict(n_top=B.MAX_TOP + 1, ids_stride=9999, teacher_stride=9999), dict(temperature=0.0),
                dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(label_weight=math.nan), dict(teacher_weight=math.inf), dict(d_row_weight=P + 2),
                dict(d_loss=0), dict(d_loss=P + 2), dict(d_dz=P + 1), dict(dz_stride=49),
                dict(dz_stride=51)):
        _refused(B.distill, *{**good, **bad}.values())
    size = B.distill_workspace(2, 100000, 4)                  # few rows, cut into parts
    long = dict(n_tokens=2, n_vocabulary=100000, z_stride=100000, dz_stride=100000, d_workspace=P, workspace_bytes=size)
    assert size > 0 and B.distill_workspace(9, 50, 4) == 0 and B.lib().mgwfbp_distill_workspace(1, 1, 1, None) == -1
    for bad in (dict(d_workspace=0), dict(d_workspace=P + 128), dict(workspace_bytes=size - 1)):
        _refused(B.distill, *{**good, **long, **bad}.values())
    for bad in ((-1, 5, 0), (1, 0, 0), (1, 5, -1), (1, 5, B.MAX_TOP + 1)):
        _refused(B.distill_workspace, *bad)
    B.distill(*{**good, "n_tokens": 0, "d_z": 0, "d_loss": 0, "d_ids": 0}.values())


def test_the_structure_of_sequences_is_the_headers():
    assert C.sizeof(B.Sequences) == 32 and B.Sequences.d_offsets.offset == 16 and B.Sequences.offset_type.offset == 24 and B.RECUR_BLOCK == 128 and B.MAX_TOP == 1024


Z = torch.zeros


@pytest.mark.parametrize("call", [
    lambda: layers.norm(Z(4, 8)),                                                                # not on a GPU
    lambda: layers.norm(Z(4, 8, dtype=torch.float64)),
    lambda: layers.norm(Z(8)),
    lambda: layers.norm(Z(4, 8), Z(7)),
    lambda: layers.norm(Z(4, 8), h=Z(4, 8)),
    lambda: layers.norm(Z(4, 8), residual=Z(4, 7)),
    lambda: layers.norm(Z(4, 8), residual=Z(4, 8), h=Z(4, 8, dtype=torch.float16)),
    lambda: layers.norm(Z(4, 8), kept=layers.norm_empty(4, 9, "cpu")),
    lambda: layers.norm(Z(4, 8), kept=layers.Norm8(layers.act_empty(4, 8, "cpu"), Z(4), layers.act_empty(4, 8, "cpu"))),      # two memories of q
    lambda: layers.norm_backward(layers.norm_empty(4, 8, "cpu"), Z(4, 8)),
    lambda: layers.norm_backward(layers.norm_empty(4, 8, "cpu"), Z(4, 9)),
    lambda: layers.norm_backward(layers.norm_empty(4, 8, "cpu")._replace(rstd=Z(5)), Z(4, 8)),
    lambda: layers.recur(Z(4, 8), Z(4, 8)),
    lambda: layers.recur(Z(8), Z(8)),
    lambda: layers.recur(Z(4, 8), Z(4, 9)),
    lambda: layers.recur(Z(1, 4, 8), Z(1, 4, 8), offsets=torch.tensor([0, 4])),
    lambda: layers.recur(Z(4, 8), Z(4, 8), offsets=torch.tensor([0.0, 4.0])),
    lambda: layers.recur(Z(4, 8), Z(4, 8), offsets=torch.empty(0, dtype=torch.int64)),
    lambda: layers.recur(Z(4, 8), Z(4, 8), kind="concave"),
    lambda: layers.recur_backward(Z(4, 8), Z(4, 8), Z(1, 8), Z(4, 8)),
    lambda: layers.distill(Z(4, 8)),
    lambda: layers.distill(Z(4, 0)),
    lambda: layers.distill(Z(4, 8), ids=Z(4, 2, dtype=torch.int64)),
    lambda: layers.distill(Z(4, 8), labels=Z(4)),
    lambda: layers.distill(Z(4, 8), Z(4, 2000, dtype=torch.int64), Z(4, 2000)),
])
def test_tensors_that_are_refused(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["native", "plain"])
def test_both_ways_take_and_refuse_the_same(way, monkeypatch):
    """Calls of tensors that do not fit each other, tensors that autograd follows, negated ones; and what a call has written counts as changed."""
    if way == "plain":
        for name in ("norm", "norm_backward", "recur", "recur_backward", "distill"):
            monkeypatch.setattr(layers._native, name, lambda *a: NotImplemented)
    d = "cuda"
    x, w, r = torch.randn(130, 48, device=d), torch.ones(48, device=d), torch.randn(130, 48, device=d)
    kept, y, h, dw = layers.norm_empty(130, 48), Z(130, 48, device=d), Z(130, 48, device=d), Z(48, device=d)
    states, first, loss = Z(2, 48, device=d), Z(1, 48, device=d), Z(130, device=d)
    ids, labels = torch.arange(130 * 3, device=d).view(130, 3) % 48, torch.arange(130, device=d) % 48
    calls = {
        "norm": ([x, w, r], [y, h], lambda i, o: layers.norm(i[0], i[1], residual=i[2], y=o[0], h=o[1], kept=kept)),
        "norm_backward": ([x, w, r], [y, dw], lambda i, o: layers.norm_backward(kept, i[0], i[1], dres=i[2], dh=o[0], dw=o[1])),
        "recur": ([x, r], [y, first, states], lambda i, o: layers.recur(i[0], i[1], y=o[0], last=o[1], states=o[2])),
        "recur_backward": ([x, r, states], [y, h, first], lambda i, o: layers.recur_backward(i[0], i[1], i[2], i[1], dgate=o[0], dx=o[1], dfirst=o[2])),
        "distill": ([x, r[:, :3].contiguous()], [loss, y], lambda i, o: layers.distill(i[0], ids, i[1], labels=labels, loss=o[0], dlogits=o[1])),
    }
    for name, (read, written, call) in calls.items():
        print("[blocks]", way, name, flush=True)
        before, of_read = [t._version for t in written], [t._version for t in read]
        call(read, written)
        assert all(t._version > v for t, v in zip(written, before)) and of_read == [t._version for t in read], name
        want = [t.clone() for t in written]
        for i in range(len(read)):
            followed = list(read)
            followed[i] = read[i].clone().requires_grad_(True)
            with pytest.raises(ValueError, match="autograd"):
                call(followed, written)
            with torch.no_grad():
                call(followed, written)
            wrong = list(read)
            wrong[i] = read[i].double()
            with pytest.raises(ValueError):
                call(wrong, written)
            wrong[i] = read[i][:-1]
            with pytest.raises(ValueError):
                call(wrong, written)
            wrong[i] = torch._neg_view(read[i])
            with pytest.raises(ValueError, match="negat"):
                call(wrong, written)
            wrong[i] = read[i].cpu()
            with pytest.raises(ValueError):
                call(wrong, written)
        for i in range(len(written)):
            wrong = list(written)
            wrong[i] = written[i].double()
            with pytest.raises(ValueError):
                call(read, wrong)
            wrong[i] = Z(*(n + 1 for n in written[i].shape), device=d)
            with pytest.raises(ValueError):
                call(read, wrong)
        assert all(torch.equal(a, b) for a, b in zip(want, written)), name
    over = r.clone()
    with pytest.raises(ValueError):                                      # over the residual, but with other rows
        layers.norm(x[:65], w, residual=over.view(65, 96)[:, :48], y=y[:65], h=over[:65])
    with pytest.raises(ValueError):
        layers.recur(x, r, offsets=torch.tensor([0, 130], device=d), first=first, last=first, y=y)
    for more in (dict(y=x, kept=kept), dict(residual=r, y=over, h=over), dict(residual=over, y=over, h=over)):        # y over what the codes are made of
        with pytest.raises(ValueError):
            layers.norm(x, w, **more)
    with pytest.raises(ValueError):
        layers.recur_backward(x, r, states, x, dlast=first, dfirst=first, dgate=y, dx=h)
    with pytest.raises(ValueError):
        layers.norm(x, w, y=y, kept=kept._replace(linear=layers.Act8(kept.act.q, kept.act.scale[:1], 48)))
