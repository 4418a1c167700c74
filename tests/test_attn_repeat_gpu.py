"""Attention's results depend on a call's arguments alone (paper_2307_01236_amd/block.py, on an MI355X): the same bits whatever ran before."""
import pytest
import torch

from paper_2307_01236_amd import block as bk

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def rand(*shape, seed, dtype):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def keys(B, T, K, D, dtype, cached, seed):
    """The arguments k and v: tensors, or a cache that holds them."""
    k, v = rand(B, T, K, D, seed=seed, dtype=dtype), rand(B, T, K, D, seed=seed + 1, dtype=dtype)
    if not cached:
        return k, v
    cache = bk.Kv8.zeros(B, T, K, D, dtype)
    bk.rkb_kv8_write(cache, k, v)
    return cache, None


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("D,T,G", [(64, 700, 4), (128, 700, 1), (200, 500, 5), (64, 900, 33)])
def test_rows_that_do_not_exist_change_nothing(D, T, G, cached, dtype):
    """One query with a bias is fewer rows than a workgroup of the form for few rows has.  Before it the same form runs with all of its rows, on
    all compute units, with entries that rise by hundreds towards the query: what it leaves behind must not move the maxima of the rows that exist."""
    B, K = 64, 2
    q = rand(B, 1, K * G, D, seed=1, dtype=dtype)
    k, v = keys(B, T, K, D, dtype, cached, 2)
    how = dict(causal=True, first=T - 1, bias=bk.RelBias(rand(32, K * G, seed=4, dtype=torch.float32), 128, False))
    before = torch.zeros(512, 16, 4, D, dtype=dtype, device="cuda"), keys(512, 64, 2, D, dtype, cached, 5)
    want = None
    for rise in (0.0, 1000.0, -1000.0, 50.0):
        table = (rise * torch.arange(32, 0, -1.0))[:, None].expand(32, 4).contiguous().cuda()
        bk.rkb_attn_fwd(before[0], *before[1], causal=True, first=63, bias=bk.RelBias(table, 128, False))
        o, kept = bk.rkb_attn_fwd(q, k, v, keep="full", **how)
        got = o, kept[0], kept[1]
        assert want is None or all(torch.equal(a, b) for a, b in zip(got, want)), rise
        want = got if want is None else want
