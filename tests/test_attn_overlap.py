"""Outputs of attention and of a cache's load whose elements overlap are refused, also where their extent passes 64 bits (include/rk_block.h);
on the host, before any device call."""
import pytest

from paper_2307_01236_amd import block as bk

P = 1 << 20  # a pointer-like number that is never read: the calls below refuse first

# rows of one head, and strides of 16 columns' rows, heads and sequences that lie on top of each other
OVERLAPS = [dict(rows=3, batch=16, row=16), dict(rows=(1 << 25) + 1, batch=1 << 40, row=1 << 39), dict(rows=(1 << 24) + 2, batch=1 << 40, row=1 << 39),
            dict(rows=(1 << 25) + 3, batch=(1 << 39) + 1, row=1 << 39), dict(rows=(1 << 26) + 1, batch=(1 << 39) - 1, row=1 << 38)]


@pytest.mark.parametrize("rows,batch,row", [tuple(o.values()) for o in OVERLAPS])
def test_overlapping_outputs_are_refused(rows, batch, row):
    lib = bk.load()
    o, fine = bk.CHeads(P, batch, row, 16), bk.CHeads(P, rows * 16, 16, 16)
    a = bk.CAttn(bk.RKB_BF16, 0, 2, rows, 5, 1, 1, 16, 0.25, 0, None, None, None, 0, None, 0, 0, 0, 0)
    odd = bk.CHeads(P, 5 * 24, 17, 16)  # asks for a copy, for which there is no room: no call gets further
    assert lib.rkb_attn_fwd(a, fine, odd, odd, None, fine, None, None, P, 0, None) == bk.RKB_E_NOMEM
    assert lib.rkb_attn_fwd(a, fine, odd, odd, None, o, None, None, P, 0, None) == bk.RKB_E_INVAL
    keys = bk.CHeads(P, 5 * 16, 16, 16)
    assert lib.rkb_attn_bwd(a, fine, fine, odd, odd, fine, None, P, fine, keys, keys, None, P, 0, None) == bk.RKB_E_NOMEM
    assert lib.rkb_attn_bwd(a, fine, fine, odd, odd, fine, None, P, o, keys, keys, None, P, 0, None) == bk.RKB_E_INVAL
    for k, v in ((o, fine), (fine, o)):
        assert lib.rkb_kv8_load(bk.RKB_BF16, 2, 1, 16, bk.CKv8(P, P, rows), k, v, None) == bk.RKB_E_INVAL
