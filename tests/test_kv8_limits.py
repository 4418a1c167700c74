"""How many blocks a call may write into a cache (include/rk_block.h, rkb_kv8_write): refused past the limit, on the host before any
device call, and taken at it, on an MI355X."""
import os
import re

import pytest
import torch

from paper_2307_01236_amd import block as bk

P = 1 << 20  # a pointer-like number that is never read: the calls below refuse first
MOST = 1 << 22


def touched(rows, tokens):
    """Blocks of a head that `rows` tokens may touch, as the header has it."""
    return min((rows + 62) // 32, -(-tokens // bk.RKB_GROUP))


def test_touched_is_the_most_that_any_place_touches():
    for rows in range(1, 200):
        for tokens in (1, 31, 32, 33, 64, 100, 160, 320):
            places = ((max(first, 0), min(first + rows, tokens)) for first in range(-rows + 1, tokens))
            most = max((hi - 1) // 32 - lo // 32 + 1 for lo, hi in places if lo < hi)
            assert most <= touched(rows, tokens) and (most == touched(rows, tokens) or tokens < rows + 62), (rows, tokens)


def test_the_header_names_the_limit():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rk_block.h")).read()
    assert re.search(r"At most 2\^22 blocks .* may be touched by a call", header) and "(rows + 62) / 32" in header


# batch, rows, key heads, tokens: one block too many, or as few more as the factors allow
@pytest.mark.parametrize("batch,rows,heads,tokens", [(MOST + 1, 1, 1, 32), (MOST // 64 + 1, 1, 64, 4096), (MOST // 2 + 1, 2, 1, 64), (MOST // 8 + 1, 4096, 4, 33),
                                                     (4064, 4096, 8, 4097), (1 << 28, 1 << 28, 1, 1)])
def test_more_blocks_than_a_call_takes_are_refused(batch, rows, heads, tokens):
    if batch * heads * touched(rows, tokens) <= MOST:
        batch = MOST // (heads * touched(rows, tokens)) + 1
    at = bk.CHeads(P, rows * heads * 16, heads * 16, 16)
    for counts in (None, P):
        assert bk.load().rkb_kv8_write(bk.RKB_BF16, batch, rows, heads, 16, at, at, 0, None, counts, bk.CKv8(P, P, tokens), None) == bk.RKB_E_INVAL


@pytest.mark.gpu
def test_as_many_blocks_as_a_call_takes_are_written():
    batch, heads, tokens = MOST // 64, 64, 32
    x = torch.randn(batch, 1, heads, 1, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    cache = bk.Kv8.zeros(batch, tokens, heads, 1)
    bk.rkb_kv8_write(cache, x, -x, 7)
    k, v = bk.rkb_kv8_load(cache)
    # a block of one value x: 127 * 2^(e-1) < |x|, so half a step is less than |x| / 127
    assert bool(((k[:, 7].double() - x[:, 0].double()).abs() <= x[:, 0].double().abs() / 127).all()) and torch.equal(v, -k)
    assert not k[:, :7].any() and not k[:, 8:].any()
    del cache, k, v
    x = x[:1].expand(batch + 1, -1, -1, -1)
    with pytest.raises(bk.RKBError) as e:
        bk.rkb_kv8_write(bk.Kv8.zeros(batch + 1, tokens, heads, 1), x, x)
    assert e.value.code == bk.RKB_E_INVAL
