"""Attention's scale at the ends of 32 bits (include/rk_block.h): scores are held in steps of log2, so scale log2(e) has to be a number too."""
import ctypes as C

import pytest

from paper_2307_01236_amd import block as bk


@pytest.mark.parametrize("scale,taken", [(1e-38, True), (0.125, True), (2.3e38, True), (2.37e38, False), (3.4e38, False), (float("inf"), False), (0.0, False)])
def test_scales(scale, taken):
    a, n = bk.CAttn(bk.RKB_BF16, 0, 1, 3, 5, 1, 1, 16, scale, 0, None, None, None, 0, None, 0, 0, 0, 0), C.c_size_t(0)
    want = bk.RKB_OK if taken else bk.RKB_E_INVAL
    assert bk.load().rkb_attn_fwd_workspace(a, 0, 1, n) == want and bk.load().rkb_attn_bwd_workspace(a, 0, 1, n) == want
