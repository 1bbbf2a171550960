"""The gradient operators at the ends of their ranges: values that are not finite or enormous, checkpoints in larger memory, tensors
that autograd follows, and the forms that only long calls take.  References and tolerances as in test_gpu_layers.py."""
import math

import pytest
import torch

from paper_1912_09268_amd import layers
from test_gpu_layers import DT, OWN, _close, _f64, _say

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
