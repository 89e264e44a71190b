"""Scores of the 8-bit attention where queries and keys' scales are far from 1 and their products are not: tolerances as in test_gpu_cache8."""
import numpy as np
import pytest
import torch

from test_gpu_cache8 import Case8, check_attention, run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-100, -60, 60, 98, 112])
@pytest.mark.parametrize("heads", [(8, 1, 256), (4, 2, 128), (40, 2, 128), (8, 8, 64), (16, 4, 64)], ids=lambda h: "x".join(map(str, h)))
def test_large_queries_over_keys_of_small_scales(heads, power):
    """Queries of 2^power over keys whose scales make up for it, down to the least that an append writes."""
    c = Case8(heads, 16, [300, 20, 41], [1, 5, 2], 16, seed=power + 200)
    c.scales[0] = (c.scales[0] * 2.0 ** -min(power, 91)).astype(np.float32).astype(np.float64)   # 2^-9 and more already
    q = torch.from_numpy(c.rng.normal(size=(c.rows, c.hq * c.dh)) * 2.0 ** power).cuda().bfloat16()
    q, out, lse, status = run_attention(c, q=q, scale=2.0 ** (min(power, 91) - power) * c.dh ** -0.5)
    assert status == 0
    check_attention(c, q, out, lse, scale=2.0 ** (min(power, 91) - power) * c.dh ** -0.5)


@pytest.mark.parametrize("power", [117, 122, 126])
@pytest.mark.parametrize("heads", [(8, 1, 256), (4, 2, 128), (40, 2, 128), (8, 8, 64), (16, 4, 64)], ids=lambda h: "x".join(map(str, h)))
def test_the_largest_queries_over_keys_of_the_least_scales(heads, power):
    """Scores of up to 2^40: one key takes all, and nothing passes fp32's largest on the way."""
    c = Case8(heads, 16, [300, 20, 41], [1, 5, 2], 16, seed=power)
    c.scales[0] = np.where(np.isnan(c.scales[0]), np.nan, 2.0 ** -100)
    q = torch.from_numpy(c.rng.uniform(-1.9, 1.9, (c.rows, c.hq * c.dh)) * 2.0 ** power).cuda().bfloat16()
    q, out, lse, status = run_attention(c, q=q)
    assert status == 0 and bool(out.isfinite().all()) and bool(lse[:int(c.start[-1])].isfinite().all())
    check_attention(c, q, out, lse)
