"""The norms' bounds of attention's gradients (attn_norms) on the CPU: the library's roundings stay within them, and do . o left as the kept
output gives it does not."""
import pytest
import torch

import attn_norms as an

MEANS = (3.0, 16.0)  # of keys and values


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", an.SHAPES)
def test_bounds_tell_the_correction_from_its_loss(name, dtype):
    *sizes, table = an.SHAPES[name]
    (_, _, _, do), _, case = an.case_of(*sizes, dtype, *MEANS, table=table)
    for kept in (dtype, torch.float32):
        limits = an.bounds(case, do, dtype, kept)
        right = an.errors(case, do, an.emulate(case, do, dtype, kept))
        assert all(e is None or e <= b / 2 for e, b in zip(right, limits))
        lost = an.errors(case, do, an.emulate(case, do, dtype, kept, corrected=False))
        if kept != torch.float32:  # the output in 16 bits: its rounding is most of the error
            assert lost[0] > 2 * limits[0] and (lost[3] is None or lost[3] > 1.5 * limits[3])
        if dtype == torch.bfloat16:
            assert lost[0] > 2 * limits[0] and (kept == torch.float32 or lost[1] > 2 * limits[1])


def test_bounds_are_a_few_roundings():
    """Not so wide that anything passes: dk and dv within 2.2 U of their own size (rounded on the way in and on the way out), dq (whose ds cancel the keys' mean) within seven."""
    *sizes, table = an.SHAPES["key_splits"]
    (_, _, _, do), _, case = an.case_of(*sizes, torch.bfloat16, *MEANS, table=table)
    limits = an.bounds(case, do, torch.bfloat16, torch.bfloat16)
    sizes = [float(g.norm()) for g in case.backward(do)[0]]
    u = 2.0 ** -8
    assert limits[0] < 7 * u * sizes[0] and limits[1] < 2.2 * u * sizes[1] and limits[2] < 2.2 * u * sizes[2] and limits[3] < 2 * u * sizes[3]
