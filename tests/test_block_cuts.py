"""How the block operators' products are cut (csrc/rkb_cut.h), on a host without a GPU."""
import random

import pytest

import cuts
from paper_2307_01236_amd import block as bk


@pytest.mark.parametrize("size,what", cuts.GATED_SIZES)
def test_sizes_take_the_tiles_they_are_there_for(size, what):
    """The sizes at which test_block_gpu compares every element: figures fitted anew may move
    them, and then others have to stand for these tiles."""
    got = cuts.gated(*size)._asdict()
    assert {k: got[k] for k in what} == what


def test_the_sizes_leave_no_tile_out():
    sums = {c["sums"][:2] for _, c in cuts.GATED_SIZES if "sums" in c}
    assert sums == {(256, 2), (192, 2), (128, 2), (128, 4)} and any(c.get("few") for _, c in cuts.GATED_SIZES)
    assert {c["dx"][:2] for _, c in cuts.GATED_SIZES if "dx" in c} == sums
    assert {c["dw"][:2] for _, c in cuts.GATED_SIZES if "dw" in c} == {(256, 2), (128, 2), (128, 4)}
    assert {(c["pair"][0], c["pair"][1] > 1) for _, c in cuts.GATED_SIZES if "pair" in c} == {(b, s) for b in (2, 4) for s in (True, False)}


@pytest.mark.parametrize("size,want", cuts.WEIGHT_GRAD_SIZES)
def test_weight_gradient_sizes_take_the_tiles_they_are_there_for(size, want):
    assert cuts.weight_grad(*size) == want
