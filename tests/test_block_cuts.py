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


def test_rows_of_a_tile_stay_within_32_bit_offsets():
    """A lane's place in a stage of an operand whose rows run along k is a 32-bit number of bytes from the tile's first
    row: the last row's last chunk must not pass it, over all widths that the calls take.  The longest rows are
    copies in the workspace and dg and du, whose columns are rounded up to 8."""
    rng, longest = random.Random(3), bk.RKB_MAX_COLS

    def reaches(tile_rows, columns):
        return (tile_rows - 1) * (-(-columns // 8) * 8) * 2 + 7 * 16 < 1 << 32

    sizes = [(256, 1024, 8421512), (512, 512, longest), (200, longest, 64), (8192, longest, 8192), (8192, 8192, longest)]
    sizes += [tuple(round(2 ** rng.uniform(0, top)) for top in (14, 24, 24)) for _ in range(20000)]
    assert any(not reaches(256, f) for _, _, f in sizes)  # a case for the choice
    for rows, width, hidden in sizes:
        c = cuts.gated(rows, width, hidden)
        assert reaches(c.sums.rows, width) and reaches(c.dx.rows, hidden), (rows, width, hidden)
        assert reaches(128, width) and reaches(128, hidden)  # wg and wu beside x, and dg and du in a launch with the weights' gradients
