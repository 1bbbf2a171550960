"""Cross entropy and divergence from a teacher's top logits, with the logits' gradient, against plain 64-bit implementations.

Tolerances, u = 2^-24: an exponent's argument is a difference (one rounding) times a constant (two more), so exp(z - max) is off by 3 u |z - max| + 4 u
of itself; a sum of V of them over a workgroup's lanes by at most V / 64 + 20 roundings more; their quotient by both."""
import math

import pytest
import torch

from paper_1912_09268_amd import layers_binding as M
from paper_1912_09268_amd import layers
from test_gpu_layers import BF16, DT, F16, F32, _close, _gen, _strided, _untouched

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _say(*a):
    print("[distill]", *a, flush=True)


def _reference(z, ids, teacher, labels, tau, lw, tw, rw):
    """(loss, slack, dz, slack) in 64 bits."""
    tokens, vocabulary = z.shape
    tau, lw, tw = (float(torch.tensor(v, dtype=torch.float32)) for v in (tau, lw, tw))
    z64 = z.double()
    most = z64.amax(1, keepdim=True)
    depth = (most - z64).clamp(max=200.0)                                # beyond that nothing is left of an exponential
    loss, off, dz, dz_off = z64.new_zeros(tokens), z64.new_zeros(tokens), torch.zeros_like(z64), torch.zeros_like(z64)
    rw = torch.ones(tokens, device="cuda") if rw is None else rw
    live = rw != 0
    sum_off = (vocabulary / 64 + 30) * U
    if labels is not None and lw != 0:
        there = (labels >= 0) & (labels < vocabulary) & live
        at = labels.long().clamp(0, vocabulary - 1)[:, None]
        log_q = z64 - torch.logsumexp(z64, 1, keepdim=True)
        picked = log_q.gather(1, at).squeeze(1)
        loss += torch.where(there, -lw * picked, 0.0)
        # the sum is dominated by terms near the largest: those that are off by more are small in the same measure
        mean_depth = (log_q.exp() * depth).sum(1)
        rel = sum_off + 3 * U * mean_depth
        off += torch.where(there, abs(lw) * (rel + 8 * U * (1 + picked.abs() + (most.squeeze(1) - z64.gather(1, at).squeeze(1)).abs())), 0.0).nan_to_num(posinf=0.0)
        q = log_q.exp()
        one = torch.zeros_like(q).scatter_(1, at, 1.0)
        dz += torch.where(there[:, None], lw * (q - one), 0.0)
        dz_off += torch.where(there[:, None], abs(lw) * (q * (rel[:, None] + 3 * U * depth + 8 * U) + 4 * U * one), 0.0)
    taught = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    if ids is not None and ids.shape[1] and tw != 0:
        there = (ids >= 0) & (ids < vocabulary) & (teacher != -math.inf)
        taught = there.any(1) & live
        at = ids.long().clamp(0, vocabulary - 1)
        s = torch.where(there, teacher.double() / tau, -math.inf)
        log_p = s - torch.logsumexp(s, 1, keepdim=True)
        p = torch.where(there, log_p.exp(), 0.0)
        log_r = z64 / tau - torch.logsumexp(z64 / tau, 1, keepdim=True)
        picked = log_r.gather(1, at)
        terms = torch.where(p > 0, p * (log_p - picked), 0.0)
        loss += torch.where(taught, tw * tau * tau * terms.sum(1), 0.0)
        r = log_r.exp()
        reach = torch.where(there, (s.amax(1, keepdim=True) - s).clamp(max=200.0), 0.0)
        p_rel = (ids.shape[1] + 30) * U + 3 * U * reach.amax(1)
        r_rel = sum_off + 3 * U * (r * depth / tau).sum(1)
        sizes = torch.where(p > 0, p * (2 + log_p.abs() + picked.abs() + (most - z64).gather(1, at).abs() / tau + reach), 0.0).sum(1).nan_to_num(posinf=0.0)
        off += torch.where(taught, abs(tw) * tau * tau * (sizes * (p_rel + 12 * U) + r_rel + 8 * U * (torch.log(torch.tensor(vocabulary * 1.0)) + 2)), 0.0)
        target = torch.zeros_like(r).scatter_add_(1, at, p)
        dz += torch.where(taught[:, None], tw * tau * (r - target), 0.0)
        dz_off += torch.where(taught[:, None], abs(tw) * tau * (r * (r_rel[:, None] + 3 * U * depth / tau + 8 * U) + target * (p_rel[:, None] + 8 * U)), 0.0)
    w = rw.double()
    dead = ~live
    loss, dz = torch.where(dead, 0.0, loss * w), torch.where(dead[:, None], 0.0, dz * w[:, None])
    return loss, (off * w.abs()).nan_to_num() + 1e-37, dz, (dz_off * w.abs()[:, None] + 2 * U * dz.abs()).nan_to_num() + 1e-37


def _case(tokens, vocabulary, top, dtype, seed, how="dense", teacher_t="f32", ids_t=torch.int64):
    g = _gen(seed)
    z, _ = _strided((tokens, vocabulary), DT[dtype], how)
    z.copy_(3.0 * torch.randn(tokens, vocabulary, generator=g, device="cuda"))
    ids = torch.randint(-vocabulary // 8 - 1, vocabulary + vocabulary // 8 + 1, (tokens, max(top, 1)), generator=g, device="cuda")[:, :top].to(ids_t)
    teacher = (2.0 * torch.randn(tokens, max(top, 1), generator=g, device="cuda")).sort(1, descending=True).values[:, :top].to(DT[teacher_t])
    labels = torch.randint(-2, vocabulary + 1, (tokens,), generator=g, device="cuda").to(ids_t)
    rw = torch.rand(tokens, generator=g, device="cuda")
    if tokens > 4:
        rw[3] = 0.0
    return z, ids, teacher, labels, rw


SIZES = [(1, 1, 1), (1, 131072, 64), (5, 3, 2), (7, 512, 8), (9, 513, 33), (33, 2048, 64), (8, 2049, 1), (6, 8191, 100), (5, 16385, 17), (9, 30522, 64), (4, 32769, 16),
         (3, 65536, 8), (4, 100003, 40), (3, 131073, 5), (2, 200001, 1000), (65, 1000, 0), (101, 40001, 9), (70, 66001, 3), (110, 131100, 4), (6, 1500, 65), (5, 16384, 5), (200, 20003, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.7])
@pytest.mark.parametrize("tokens,vocabulary,top", SIZES)
def test_distill(tokens, vocabulary, top, tau, dtype):
    how = "strided" if (tokens + top) % 2 else "dense"
    _say(tokens, vocabulary, top, tau, dtype, how)
    z, ids, teacher, labels, rw = _case(tokens, vocabulary, top, dtype, tokens + vocabulary, how, "bf16" if top % 3 == 1 else "f32", torch.int32 if top % 2 else torch.int64)
    for parts in ("both", "labels", "teacher"):
        i, s = (None, None) if parts == "labels" or top == 0 else (ids, teacher)
        l = None if parts == "teacher" else labels
        dz, whole = _strided((tokens, vocabulary), DT[dtype], how)
        loss = layers.distill(z, i, s, labels=l, temperature=tau, label_weight=0.3, teacher_weight=0.6, row_weight=rw, loss=torch.empty(tokens, device="cuda"), dlogits=dz)
        want, off, want_dz, dz_off = _reference(z, i, s, l, tau, 0.3, 0.6, rw)
        _close(loss, want, off, f"loss, {parts}")
        _close(dz, want_dz, dz_off, f"dz, {parts}")
        assert _untouched(dz, whole, math.nan)
        assert torch.equal(layers.distill(z, i, s, labels=l, temperature=tau, label_weight=0.3, teacher_weight=0.6, row_weight=rw), loss)
        over = z.clone()
        layers.distill(over, i, s, labels=l, temperature=tau, label_weight=0.3, teacher_weight=0.6, row_weight=rw, dlogits=over)
        assert torch.equal(over, dz)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocabulary", [300, 5000, 140000])
def test_the_same_index_twice(vocabulary, dtype):
    _say("twice", vocabulary, dtype)
    z, _, teacher, _, _ = _case(6, vocabulary, 12, dtype, 3)
    ids = torch.tensor([4, 7, 4, 4, 9, 7, 0, vocabulary - 1, 4, 0, -1, 9], device="cuda").expand(6, 12).contiguous()
    labels = torch.tensor([4, 7, 1, vocabulary - 1, -1, 0], device="cuda")
    dz = torch.empty_like(z)
    loss = layers.distill(z, ids, teacher, labels=labels, temperature=1.5, dlogits=dz)
    want, off, want_dz, dz_off = _reference(z, ids, teacher, labels, 1.5, 1.0, 1.0, None)
    _close(loss, want, off, "loss")
    _close(dz, want_dz, dz_off + 12 * U, "dz")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocabulary", [40, 3000, 140001])
def test_rows_that_ask_for_nothing_and_values_that_are_not_finite(vocabulary, dtype):
    _say("masks", vocabulary, dtype)
    tokens, top = 12, 4
    z, _, teacher, labels, _ = _case(tokens, vocabulary, top, dtype, 9)
    ids = torch.randint(0, vocabulary, (tokens, top), generator=_gen(4), device="cuda")
    ids[:, 1] = (ids[:, 0] + 1) % vocabulary
    labels = torch.randint(0, vocabulary, (tokens,), generator=_gen(5), device="cuda")
    rw = torch.ones(tokens, device="cuda")
    rw[0] = 0.0
    z[0] = math.nan                                                      # padded: not looked at
    z[1], labels[1], ids[1] = math.inf, -1, -1                           # neither label nor entry
    labels[2], teacher[2] = -1, -math.inf                                # all entries without probability
    teacher[3, 1:] = -math.inf
    z[4, : vocabulary // 2], labels[4], ids[4] = -math.inf, vocabulary - 1, torch.arange(vocabulary - 4, vocabulary, device="cuda")      # masked places
    z[5, 7], labels[5], ids[5] = -math.inf, 7, torch.tensor([8, 9, 10, 11], device="cuda")     # a label that cannot be: infinite loss, finite gradient
    z[6, 3] = math.nan
    z[7, 3] = math.inf
    teacher[8, 0] = math.nan
    z[9] = -math.inf
    z[10] = torch.finfo(DT[dtype]).min                                   # masked by the type's lowest value, but for two places
    z[10, 5], z[10, 6], labels[10], ids[10] = 1.0, 2.0, 5, torch.tensor([5, 6, -1, -1], device="cuda")
    dz = torch.empty_like(z)
    loss = layers.distill(z, ids, teacher, labels=labels, temperature=2.0, row_weight=rw, dlogits=dz)
    torch.cuda.synchronize()
    for t in (0, 1, 2):
        assert float(loss[t]) == 0.0 and not bool(dz[t].any()), t
    want, off, want_dz, dz_off = _reference(z, ids, teacher, labels, 2.0, 1.0, 1.0, rw)
    for t in (3, 4, 10, 11):
        assert math.isfinite(float(want[t]))
        _close(loss[t:t + 1], want[t:t + 1], off[t:t + 1], f"loss {t}")
        _close(dz[t:t + 1], want_dz[t:t + 1], dz_off[t:t + 1], f"dz {t}")
    assert not bool(dz[4, : vocabulary // 2].any())
    assert float(loss[5]) == math.inf and bool(dz[5].isfinite().all())
    _close(dz[5:6], want_dz[5:6], dz_off[5:6], "dz 5")
    for t in (6, 7, 9):
        assert math.isnan(float(loss[t])) and bool(dz[t].isnan().all()), t
    assert math.isnan(float(loss[8])) and bool(dz[8, ids[8]].isnan().any())
    # weights of zero leave their part out, whatever is in it
    loss = layers.distill(z, ids, teacher, labels=labels, label_weight=0.0, teacher_weight=0.0, dlogits=dz)
    assert not bool(loss.any()) and not bool(dz.any())


def test_enormous_logits():
    z = torch.tensor([[3e38, 1e38, -3e38, 0.0], [-3e38, -3e38, -1e38, -3e38], [3e38, 3e38, 0.0, 1.0]], device="cuda")
    dz = torch.empty_like(z)
    loss = layers.distill(z, labels=torch.tensor([0, 2, 1], device="cuda"), dlogits=dz)
    assert torch.allclose(loss, torch.tensor([0.0, 0.0, math.log(2.0)], device="cuda"), rtol=4e-7, atol=0)
    assert torch.allclose(dz, torch.tensor([[0.0] * 4, [0.0] * 4, [0.5, -0.5, 0.0, 0.0]], device="cuda"), atol=2e-7)


def test_gradient_against_differences():
    g = _gen(2)
    z, ids, teacher, labels, rw = _case(8, 50, 6, "f32", 21)
    dz = torch.empty_like(z)
    layers.distill(z, ids, teacher, labels=labels, temperature=1.7, label_weight=0.4, row_weight=rw, dlogits=dz)

    def total(z):
        return float(layers.distill(z, ids, teacher, labels=labels, temperature=1.7, label_weight=0.4, row_weight=rw).double().sum())

    e = 2.0 ** -6
    for seed in range(5):
        v = torch.randn(z.shape, generator=_gen(30 + seed), device="cuda")
        along = (total(z + e * v) - total(z - e * v)) / (2 * e)
        # eight rows' losses of about 10, off by some 20 u each, over 2 e; the third derivative of a row's loss along v is below 20 |v|^3 / tau
        assert abs(along - float((dz.double() * v.double()).sum())) < 8 * 10 * 20 * U / e + e * e / 6 * 8 * 200


def test_offsets_beyond_32_bits_and_strides_of_top_entries():
    _say("offsets beyond 2^32 elements")
    rows, stride, vocabulary = 530000, 8192, 40
    memory = torch.zeros(rows * stride, dtype=BF16, device="cuda")
    z = torch.as_strided(memory, (rows, vocabulary), (stride, 1))
    z[-100:] = torch.randn(100, vocabulary, generator=_gen(1), device="cuda").to(BF16)
    wide_ids, wide = torch.randint(0, vocabulary, (rows, 9), generator=_gen(2), device="cuda"), torch.randn(rows, 11, generator=_gen(3), device="cuda")
    ids, teacher = wide_ids[:, 2:5], wide[:, 4:7]                        # the first few of more
    dz = torch.empty(100, vocabulary, dtype=BF16, device="cuda")
    few = layers.distill(z[-100:].contiguous(), ids[-100:].contiguous(), teacher[-100:].contiguous(), temperature=2.0, dlogits=dz)
    loss = layers.distill(z, ids, teacher, temperature=2.0, dlogits=z)
    assert torch.equal(loss[-100:], few) and torch.equal(z[-100:], dz)


def test_no_rows_and_captured():
    empty = torch.empty(0, 10, device="cuda")
    assert layers.distill(empty, labels=torch.empty(0, dtype=torch.int64, device="cuda"), dlogits=empty).shape == (0,)
    z, ids, teacher, labels, rw = _case(20, 3000, 8, "bf16", 2)
    loss, dz = torch.empty(20, device="cuda"), torch.empty_like(z)

    def step():
        layers.distill(z, ids, teacher, labels=labels, temperature=2.0, row_weight=rw, loss=loss, dlogits=dz)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for replay in range(4):
        z.copy_(torch.randn(z.shape, generator=_gen(replay), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = loss.clone(), dz.clone()
        loss.zero_(), dz.zero_()
        step()
        assert torch.equal(got[0], loss) and torch.equal(got[1], dz), replay
