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
