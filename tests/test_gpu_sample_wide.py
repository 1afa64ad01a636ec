"""Drawn tokens where logits span the type's whole range and temperatures are as large: differences of logits, and temperatures times the logarithm of
the smallest weight, pass the largest fp32."""
import numpy as np
import pytest
import torch

import operators_oracle as oo
from paper_2203_16487_amd import binding as sd
from test_gpu_sample import check, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 4000, 12000])
def test_wide_logits_at_large_temperatures(ctx, dtype, V):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(V)
    rng = np.random.default_rng(V)
    largest = torch.finfo(dtype).max
    spread = (torch.rand((3, V), generator=gen, device="cuda") * 2 - 1) * largest
    two = torch.where(torch.rand(V, generator=gen, device="cuda") < 0.5, largest, -largest)        # half of them as large, half as small as can be
    rows = torch.stack([spread[0], two, spread[1].masked_fill(spread[2] > 0, -INF), spread[2] * 2 ** -20, spread[2].clamp(max=0)]).to(dtype)
    for T in (INF, 3.4e38, 2e37, 1.3e37, 1.2e37, 1e36, 1e30):
        for top_k, top_p, min_p in ((0, 1.0, 0.0), (0, 0.9, 0.0), (0, 0.4, 0.0), (V // 2, 1.0, 0.0), (V * 9 // 10, 0.95, 0.0), (150, 0.9, 0.0), (0, 1.0, 0.3), (0, 0.97, 0.6)):
            n = len(rows)
            check(ctx, rows, np.full(n, T, np.float32), np.full(n, top_k, np.int32), np.full(n, top_p, np.float32), np.full(n, min_p, np.float32),
                  rng.random(n).astype(np.float32))
