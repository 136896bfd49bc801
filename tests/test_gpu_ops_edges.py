"""Edges of the training-step operators: statistics at the edge of 32 bits."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2412_12487_amd as E
from tests import opsref as R

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, mean=0.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


# rows that leave lanes of their team idle, whole pieces and cut ones, from the narrowest team to past the widest
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [5, 104, 101, 904, 1001, 1600, 1501, 3200, 3001, 5600, 5003, 7200, 7001, 10400, 10001, 15200, 15001,
                                  20003])
def test_layer_norm_grad_where_mean_times_rstd_passes_32_bits(cols, dtype):
    """A constant row of 2^120 has finite statistics, and n = 0 throughout: its gradient is rstd * (g - mean(g)), although
    2^120 / sqrt(1e-5 * 2^-20) is no 32-bit number."""
    g = _gen(cols)
    x, w = _normal(g, 5, cols, dtype=dtype), _normal(g, cols, std=0.2, mean=1.0, dtype=dtype)
    dy, dr = _normal(g, 5, cols, std=0.5, dtype=dtype), _normal(g, 5, cols, dtype=dtype)
    s = E.layer_norm(x, w, None)
    x[2], s["mean"][2], s["rstd"][2] = 2.0 ** 120, 2.0 ** 120, 1024 / math.sqrt(1e-5)
    assert math.isinf(float(s["mean"][2] * s["rstd"][2]))
    out = E.layer_norm_grad(dy, x, w, s["mean"], s["rstd"], grad_residual=dr, dtype=F32)
    for k, (v, e) in R.layer_norm_grad(dy, x, w, s["mean"], s["rstd"], dr).items():
        R.close(out[k], v, e, k)
