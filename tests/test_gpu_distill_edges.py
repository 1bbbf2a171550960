"""The loss where a single lane, element or entry decides: entries that other lanes hold, and logits at the ends of what lanes, parts and rows have in common."""
import math
import os
import re

import pytest
import torch

from paper_1912_09268_amd import layers
from test_gpu_distill import _case, _reference
from test_gpu_layers import DT, _close, _gen

U = 2.0 ** -24


def _say(*a):
    print("[distill]", *a, flush=True)


def test_a_single_wavefront_waits_for_its_entries():
    """Entries lie in LDS, written by a lane each and compared by all; workgroup_all has a barrier only where there are several wavefronts."""
    source = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1912_09268_amd", "csrc", "distill.hip")).read()
    assert "if constexpr (THREADS > 64) {" in source
    assert re.search(r"void find_again\(int top\) \{\s*if constexpr \(THREADS == 64\) __syncthreads\(\);", source)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocabulary,top", [(40, 64), (300, 7), (512, 130), (1000, 64), (2048, 33), (2048, 65)])
def test_the_same_index_in_other_lanes(vocabulary, top, dtype):
    """Every index stands at least twice, in the first and the last lanes, and so does the label's."""
    _say("other lanes", vocabulary, top, dtype)
    tokens = 50
    z, _, teacher, _, _ = _case(tokens, vocabulary, top, dtype, vocabulary + top)
    half = torch.randint(0, vocabulary, (tokens, (top + 1) // 2), generator=_gen(top), device="cuda")
    ids = torch.cat([half, half.flip(1)], 1)[:, :top].contiguous()
    labels = ids[:, 0].contiguous()
    dz = torch.empty_like(z)
    loss = layers.distill(z, ids, teacher, labels=labels, temperature=1.5, dlogits=dz)
    want, off, want_dz, dz_off = _reference(z, ids, teacher, labels, 1.5, 1.0, 1.0, None)
    _close(loss, want, off, "loss")
    _close(dz, want_dz, dz_off + top * U, "dz")


def _plain(z, ids, teacher, labels, tau):
    """Loss and gradient in 64 bits, of rows that all have a label and entries."""
    with torch.enable_grad():
        z64 = z.double().requires_grad_(True)
        p = torch.log_softmax(teacher.double() / tau, 1)
        r = torch.log_softmax(z64 / tau, 1).gather(1, ids)
        loss = 0.4 * torch.nn.functional.cross_entropy(z64, labels, reduction="none") + 0.7 * tau * tau * (p.exp() * (p - r)).sum(1)
        return loss.detach(), torch.autograd.grad(loss.sum(), z64)[0]


def _places(vocabulary):
    """Where an element is the first or the last of a vector, a lane's, a part's or the row."""
    some = {0, 7, 8, *(vocabulary - k for k in (1, 2, 7, 8, 9, 15, 16, 17))}
    for border in (512, 2048, 4096, 8192, 16384, 32768):
        for last in {border, vocabulary // border * border}:
            some |= {last - 9, last - 8, last - 1, last, last + 1, last + 7, last + 8}
    return sorted(p for p in some if 0 <= p < vocabulary)


# rows (0: as many as places), logits: every form and shape, rows that end with a whole vector and such that do not
FORMS = [(0, 8), (0, 9), (0, 511), (0, 512), (0, 513), (0, 1995), (0, 2048), (0, 2049), (0, 8191), (0, 8193), (0, 16383), (0, 16390), (0, 30522), (70, 32767),
         (70, 40001), (70, 65535), (101, 100003), (101, 131071), (101, 131100), (210, 200001),                           # registers, and taken up twice
         (3, 32769), (30, 32770), (39, 40001), (60, 66001), (16, 66007), (97, 100003), (100, 131073), (90, 200001), (100, 200005)]      # parts of one vector a lane and more


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocabulary", FORMS)
def test_logits_that_decide_at_every_border(rows, vocabulary, dtype):
    """Of a row two logits make up the softmax, one of them at a border: an element that is taken twice, or left out, changes loss and gradient by a tenth and
    more.  All others are some 60 below: e^-30 each at tau = 2, 2e-8 of 200000 of them, so their errors do not count.

    A lane adds at most V / 1024 or, with rows in registers or parts, 128 numbers, and 40 more are joined; exponents are of differences near 0 for the two that
    count, and logarithms and differences of up to 100 have a few roundings."""
    _say("borders", rows, vocabulary, dtype)
    places = _places(vocabulary)
    for begin in range(0, len(places) if rows else 1, rows or 1):
        at = torch.tensor(places[begin:begin + rows] if rows else places, device="cuda")
        tokens = rows or len(places)
        at = at.repeat(-(-tokens // at.numel()))[:tokens]
        g = _gen(vocabulary + begin)
        z = (torch.rand(tokens, vocabulary, generator=g, device="cuda") - 45.0).to(DT[dtype])
        row = torch.arange(tokens, device="cuda")
        other = torch.where(at == vocabulary // 3, vocabulary // 2, vocabulary // 3)
        z[row, other] = 15.0
        z[row, at] = 15.25
        third = (at + other + 1) % vocabulary
        labels = torch.where(row % 3 == 0, at, torch.where(row % 3 == 1, other, third))
        ids = torch.stack([at, other, third, labels], 1)                  # the label's index again, so three of the rows' entries are twice there
        teacher = torch.randn(tokens, 4, generator=g, device="cuda")
        sums = (max(vocabulary / 1024, 128) + 40) * U
        for tau in (1.0, 2.0):
            want, want_dz = _plain(z, ids, teacher, labels, tau)
            dz = torch.empty_like(z)
            loss = layers.distill(z, ids, teacher, labels=labels, temperature=tau, label_weight=0.4, teacher_weight=0.7, dlogits=dz)
            size = 0.4 + 0.7 * tau * tau
            _close(loss, want, size * (2 * sums + 8 * U * 200), f"loss {tau}")
            _close(dz, want_dz, size * 2 * (sums + 40 * U), f"dz {tau}")
            assert torch.equal(layers.distill(z, ids, teacher, labels=labels, temperature=tau, label_weight=0.4, teacher_weight=0.7), loss)
            over = z.clone()
            layers.distill(over, ids, teacher, labels=labels, temperature=tau, label_weight=0.4, teacher_weight=0.7, dlogits=over)
            assert torch.equal(over, dz)


@pytest.mark.gpu
@pytest.mark.parametrize("tau", [2.0 ** -20, 2.0 ** -6, 0.25, 16.0, 1024.0, 2.0 ** 20])
@pytest.mark.parametrize("vocabulary,top", [(6, 6), (64, 64), (1000, 1000), (30522, 64)])
def test_temperatures_from_cold_to_hot(vocabulary, top, tau):
    """Entries that cover the vocabulary, where the divergence nears 0 as tau grows, and some of it: the loss is off by roundings of numbers of log V, times tau^2."""
    _say("temperature", vocabulary, top, tau)
    tokens = 20
    z, _, teacher, labels, rw = _case(tokens, vocabulary, top, "f32", vocabulary)
    ids = torch.rand(tokens, vocabulary, generator=_gen(top), device="cuda").topk(top, 1).indices.contiguous()
    for l in (None, labels):
        dz = torch.empty_like(z)
        loss = layers.distill(z, ids, teacher, labels=l, temperature=tau, label_weight=0.3, teacher_weight=0.6, row_weight=rw, dlogits=dz)
        want, off, want_dz, dz_off = _reference(z, ids, teacher, l, tau, 0.3, 0.6, rw)
        _close(loss, want, off, "loss")
        _close(dz, want_dz, dz_off, "dz")
