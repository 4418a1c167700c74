"""Which form of attention's forward takes a call (csrc/rkb_attn_cut.h, asked on the host), and that the form for few queries holds for every
number of heads that share a key head (on an MI355X)."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import attn_oracle as ao
import cuts
from paper_2307_01236_amd import block as bk

BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def few(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("cut") / "attn_cut_query.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", cuts.CSRC, os.path.join(cuts.HERE, "attn_cut_query.cpp"),
                    "-o", out], check=True)
    lib = C.CDLL(out)
    lib.few_queries_win.argtypes = [C.c_int64, C.c_int64, C.c_int]
    return lambda queries, columns, bias: bool(lib.few_queries_win(queries, columns, bias))


# 16 sequences of 4096 tokens, 4 key heads, bf16 on an MI355X: columns, a bias, heads that share a key head, queries, us by the form for few and for many
MEASURED = [(128, 0, 4, 1, 35, 68), (128, 0, 4, 16, 38, 67), (128, 0, 4, 24, 53, 68), (128, 0, 4, 32, 54, 68), (128, 0, 4, 40, 84, 71), (128, 0, 1, 64, 39, 34),
            (128, 0, 1, 96, 56, 37), (128, 0, 16, 8, 54, 225), (128, 0, 16, 32, 165, 232), (128, 0, 16, 64, 329, 249), (128, 0, 64, 1, 38, 839), (128, 0, 64, 4, 85, 845),
            (128, 0, 64, 24, 481, 891), (128, 1, 4, 16, 49, 70), (128, 1, 4, 40, 102, 75), (128, 1, 8, 4, 43, 122), (256, 0, 8, 16, 151, 283), (256, 0, 4, 40, 265, 171),
            (64, 0, 4, 32, 27, 50), (64, 0, 4, 64, 37, 54), (64, 0, 4, 96, 63, 55), (64, 0, 16, 48, 105, 162), (64, 1, 4, 24, 46, 54), (64, 1, 4, 64, 72, 57)]


@pytest.mark.parametrize("columns,bias,group,queries,us_few,us_many", MEASURED)
def test_the_faster_form_is_taken(few, columns, bias, group, queries, us_few, us_many):
    assert few(queries, columns, bias) == (us_few < us_many)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,Q,T,H,K,D,more", [
    (2, 20, 300, 16, 2, 96, {}), (1, 1, 700, 128, 1, 64, dict(bias=(32, 128, False, FP), causal=True, firsts=699)), (2, 32, 130, 21, 3, 128, dict(mask=True)),
    (1, 31, 90, 65, 1, 40, dict(causal=True, firsts=[50])), (3, 7, 600, 12, 2, 200, dict(lens=[600, 33, 0])), (2, 64, 257, 6, 2, 64, dict(lens=[257, 100], mask=True)),
    (2, 12, 150, 18, 2, 72, dict(bias=(16, 60, True, None), lens=[150, 70]))])
def test_heads_that_share_keys_fill_many_workgroups(B, Q, T, H, K, D, more, dtype):
    """More than 64 rows of a key head by the form for few queries: forward from tensors and from a cache, and the gradients after it."""
    from test_attn_gpu import check_step, problem

    more = dict(more)
    if more.get("bias") and more["bias"][3] is None:
        more["bias"] = more["bias"][:3] + (dtype,)
    tensors, how, case = problem(B, Q, T, H, K, D, dtype, **more)
    check_step(tensors, how, case)
    q, k, v, _ = tensors
    cache = bk.Kv8.zeros(B, T, K, D, dtype)
    bk.rkb_kv8_write(cache, k, v)
    want, kept = bk.rkb_attn_fwd(q, *bk.rkb_kv8_load(cache), keep="full", **how)
    got, kept8 = bk.rkb_attn_fwd(q, cache, keep="full", **how)
    assert torch.equal(got, want) and torch.equal(kept[0], kept8[0]) and torch.equal(kept[1], kept8[1])


@pytest.mark.gpu
@pytest.mark.parametrize("columns", [64, 128])
def test_both_forms_next_to_the_border_agree(columns):
    """The last query of a call that the form for few takes and of one more, which goes to the other: within both forms' bounds of the definition."""
    border = 64 if columns == 64 else 32
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen).to(BF)  # noqa: E731
    q, k, v = r(1, border + 1, 4, columns), r(1, 200, 2, columns), r(1, 200, 2, columns)
    case = ao.Case(q, k, v)
    want, bound = case.forward()[0], case.forward_bounds(BF)[0]
    for n in (border, border + 1):
        o = bk.rkb_attn_fwd(q[:, :n].cuda(), k.cuda(), v.cuda())[0]
        assert ao.worst(o, want[:, :n], bound[:, :n]) <= 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Q", [31, 32, 33, 50, 64, 65])
def test_a_cache_takes_the_form_that_its_values_take(Q, D):
    """The same bits over a cache and over what it stands for, on both sides of the rule's borders."""
    gen = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=gen).to(BF).cuda()  # noqa: E731
    q, cache = r(2, Q, 4, D), bk.Kv8.zeros(2, 300, 4, D)
    bk.rkb_kv8_write(cache, r(2, 300, 4, D), r(2, 300, 4, D))
    assert torch.equal(bk.rkb_attn_fwd(q, cache)[0], bk.rkb_attn_fwd(q, *bk.rkb_kv8_load(cache))[0])
