"""Attention's gradients as a whole (paper_2307_01236_amd/block.py, on an MI355X) against their 64-bit definition, by the norms that
independent roundings give (attn_norms): where keys and values have means, an error of do . o would be the largest of all."""
import pytest
import torch

import attn_norms as an
from paper_2307_01236_amd import block as bk

pytestmark = pytest.mark.gpu
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("keep", ["none", "16bit", "full"])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("name", an.SHAPES)
def test_gradients_are_within_a_few_roundings(name, dtype, keep):
    *sizes, table = an.SHAPES[name]
    (q, k, v, do), more, case = an.case_of(*sizes, dtype, 3.0, 16.0, table=table)
    how = dict(bias=bk.RelBias(more["table"].cuda(), more["max_distance"], more["two_sided"])) if table else {}
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    _, kept = bk.rkb_attn_fwd(q, k, v, keep=keep, **how)
    got = bk.rkb_attn_bwd(do.cuda(), q, k, v, kept, **how)
    limits = an.bounds(case, do, dtype, dtype if keep == "16bit" else FP)
    for what, error, limit in zip(("dq", "dk", "dv", "dtable"), an.errors(case, do, got), limits):
        assert (error is None) == (limit is None) and (error is None or error <= limit), (what, error, limit)
