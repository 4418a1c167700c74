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


# queries, keys, heads, key heads, width, type, over a cache, what else: the form for few rows and the one for many, keys (and for gradients
# queries) in splits or whole
FORMS = {
    "few": (1, 300, 8, 2, 64, HF, False, {}), "few_splits": (2, 1500, 8, 2, 128, BF, False, {}), "few_bias": (1, 700, 6, 2, 72, HF, False, dict(bias=True)),
    "few_cache": (1, 400, 16, 4, 128, BF, True, {}), "few_cache_splits": (3, 2000, 4, 4, 64, HF, True, dict(bias=True, causal=True, first=1997)),
    "many": (150, 260, 4, 2, 64, HF, False, dict(bias=True)), "many_splits": (130, 700, 4, 2, 128, BF, False, dict(causal=True, first=500)),
    "many_cache": (200, 300, 2, 2, 40, BF, True, {}), "many_queries": (600, 90, 4, 2, 64, BF, False, dict(bias=True)), "wide": (70, 600, 2, 1, 256, HF, False, {}),
}


def steps(q, k, v, do, how):
    """Output, log-sums and, where keys are no cache, gradients."""
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="full", **how)
    out = [o, kept[0], kept[1]]
    return out if v is None else out + [g for g in bk.rkb_attn_bwd(do, q, k, v, kept, **how) if g is not None]


def of_form(name, B):
    Q, T, H, K, D, dtype, cached, more = FORMS[name]
    more = dict(more)
    q, do = rand(B, Q, H, D, seed=1, dtype=dtype), rand(B, Q, H, D, seed=2, dtype=dtype)
    k, v = keys(B, T, K, D, dtype, cached, 3)
    if more.pop("bias", False):
        more["bias"] = bk.RelBias(rand(32, H, seed=6, dtype=torch.float32), 128, not more.get("causal", False))
    return q, k, v, do, more


@pytest.mark.parametrize("name", FORMS)
def test_the_same_call_gives_the_same_bits(name):
    """Again and again, whatever other forms ran between."""
    q, k, v, do, how = of_form(name, 3)
    first = steps(q, k, v, do, how)
    for other in FORMS:
        steps(*of_form(other, 5))
        assert all(torch.equal(a, b) for a, b in zip(first, steps(q, k, v, do, how))), other


@pytest.mark.parametrize("name", FORMS)
def test_a_sequence_alone_is_what_it_is_in_a_batch_with_the_same_splits(name):
    """Sums are cut by how many workgroups a call has; these calls have so few, alone and in a batch of three, that as much as the keys' (and queries')
    number allows is cut off either way."""
    q, k, v, do, how = of_form(name, 3)
    together = steps(q, k, v, do, how)
    for b in range(3):
        one = lambda t: t[b:b + 1]  # noqa: E731
        if v is None:
            alone = bk.Kv8(k.codes[:, b:b + 1].contiguous(), k.exps[:, b:b + 1].contiguous(), (1, *k.shape[1:]), k.dtype), None
        else:
            alone = one(k), one(v)
        got = steps(one(q), *alone, one(do), how)
        # all but the table's gradient, which is of all sequences
        assert all(torch.equal(one(a), g) for a, g in list(zip(together, got))[:6])
