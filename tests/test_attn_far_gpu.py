"""Bias gradients whose last bucket begins past 128 positions (paper_2307_01236_amd/block.py, on an MI355X), for heads of more than 64
columns: kernels of their own, whose diagonals LDS holds fewer of at a time."""
import pytest
import torch

import attn_oracle as ao
from test_attn_gpu import BF, FP, HF, check_step, problem

pytestmark = pytest.mark.gpu

# B, Q, T, heads, key heads, width, what else
SHAPES = {
    "two_sides": (1, 200, 1300, 2, 1, 96, dict(bias=(128, 1024, True, FP), firsts=500)),
    "one_side": (2, 330, 700, 2, 2, 128, dict(bias=(40, 600, False, None), causal=True, firsts=[370, 100])),
    "masked": (2, 70, 420, 4, 2, 72, dict(bias=(40, 500, True, None), lens=[420, 200], mask=True, firsts=[100, 0])),
    "wide": (1, 130, 1100, 2, 1, 256, dict(bias=(64, 1024, True, FP), firsts=400)),
    "wide_odd": (2, 97, 400, 2, 2, 137, dict(bias=(34, 700, False, None), causal=True, firsts=[300, 350], lens=[400, 390])),
    "wide_queries": (1, 700, 90, 4, 1, 160, dict(bias=(60, 800, True, FP), firsts=-300)),
}


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("name", SHAPES)
def test_step(name, dtype):
    *sizes, more = SHAPES[name]
    more = dict(more)
    more["bias"] = more["bias"][:3] + (more["bias"][3] or dtype,)
    buckets, distance, two_sided, _ = more["bias"]
    last = (buckets // 2 if two_sided else buckets) - 1
    assert sizes[5] > 64 and ao.bucket(-128, buckets, distance, two_sided) < last  # what this is here for
    check_step(*problem(*sizes, dtype, **more))
