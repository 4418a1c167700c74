"""The block operators at sizes that take every tile, split and launch (cuts.GATED_SIZES), and layer norm's
column sums over many rows in turn, element by element against the 64-bit definitions within the bounds that
32-bit sums and one rounding of each output (and of dg and du) allow; the 64-bit side runs on the GPU."""
import math

import pytest
import torch

import block_oracle as bo
import cuts
from paper_2307_01236_amd import block as bk

pytestmark = pytest.mark.gpu
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def normal(gen, *shape, dtype, scale=1.0):
    return torch.randn(*shape, generator=gen, device="cuda").mul_(scale).to(dtype)


def worst(got, ref, bound):
    """Largest error over its bound (NaN counts as infinite)."""
    return float(torch.nan_to_num((got.double() - ref).abs() / bound, nan=math.inf).max())


def values(c, cols):
    """What a checkpoint's codes and exponents stand for, and its steps."""
    step = torch.exp2(c.exps.double() - 127).repeat_interleave(bk.RKB_GROUP, 1)
    assert bool((c.codes[:, cols:] == 0).all())
    return (c.codes.double() * step)[:, :cols], step[:, :cols]


@pytest.mark.parametrize("size,what", cuts.GATED_SIZES)
def test_gated_by_every_tile(size, what):
    rows, width, hidden = size
    dtype, act = ((BF, "silu"), (HF, "gelu"), (BF, "gelu"), (HF, "silu"))[cuts.GATED_SIZES.index((size, what)) % 4]
    gen = torch.Generator(device="cuda").manual_seed(11)
    x, wg, wu = (normal(gen, *s, dtype=dtype, scale=f) for s, f in (((rows, width), 1.0), ((hidden, width), width ** -0.5),
                                                                    ((hidden, width), width ** -0.5)))
    dh = normal(gen, rows, hidden, dtype=dtype, scale=0.1)
    X, G, U, DH = x.double(), wg.double(), wu.double(), dh.double()
    h_ref, g_ref, u_ref = bo.gated(X, G, U, act)
    h_bound, eg, eu = bo.gated_bounds(X, G, U, act, dtype)
    first = again = None
    for keep in ("none", "full", "16bit", "8bit"):
        h, kept = bk.rkb_gated_fwd(x, wg, wu, act, keep=keep)
        assert worst(h, h_ref, h_bound) <= 1.0, keep
        assert first is None or torch.equal(h, first), keep
        first = h
        g, u, slack = g_ref, u_ref, (eg, eu)
        if keep in ("full", "16bit"):
            kind = FP if keep == "full" else dtype
            for t, ref, e in zip(kept, (g_ref, u_ref), (eg, eu)):
                assert t.dtype == kind and worst(t, ref, e + bo.rounding(ref, kind) * 1.01) <= 1.0, keep
            g, u, slack = kept[0].double(), kept[1].double(), (0.0, 0.0)
        elif keep == "8bit":
            g, u = (values(c, hidden)[0] for c in kept)
            for v, c, ref, e in zip((g, u), kept, (g_ref, u_ref), (eg, eu)):
                assert worst(v, ref, values(c, hidden)[1] / 2 + 2 * e) <= 1.0, keep
            slack = (0.0, 0.0)
        got = bk.rkb_gated_bwd(dh, x, wg, wu, act, kept, want_h=True)
        refs = bo.gated_grads(DH, X, G, U, act, g, u)
        for name, t, ref, e in zip(("dx", "dwg", "dwu", "h"), got, refs,
                                   bo.gated_grad_bounds(DH, X, G, U, act, g, u, dtype, *slack)):
            assert worst(t, ref, e) <= 1.0, (keep, name)
            if name != "h":  # two roundings of each operand and result: rms below the bound of one
                assert float((t.double() - ref).norm() / ref.norm()) <= bo.ROUND[dtype][0], (keep, name)
        if keep == "none":
            again = got
        elif keep == "full":  # g and u made again are the same bits as those kept in 32
            assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("size,what", cuts.WEIGHT_GRAD_SIZES)
def test_weight_gradient_by_every_tile(size, what):
    rows, n, k = size
    gen = torch.Generator(device="cuda").manual_seed(12)
    dy, x = normal(gen, rows, n, dtype=BF), normal(gen, rows, k, dtype=BF)
    c = bk.rkb_ckpt8_save(x)
    for kept, ref in ((x, x.double()), (c, bk.rkb_ckpt8_load(c).double())):
        want = torch.mm(dy.double().t().contiguous(), ref)
        bound = bo.sum_bound(torch.mm(dy.double().abs().t().contiguous(), ref.abs()), rows) + bo.rounding(want, BF)
        assert worst(bk.rkb_weight_grad(dy, kept), want, bound) <= 1.0


def test_offsets_past_31_bits_within_a_tile():
    """128 rows of the widest matrices, which lie 2^24 elements apart in the workspace: x in the forward, dg and du in the
    backward.  One element of each row is not zero, so that every result is one known number."""
    rows, wide = 128, bk.RKB_MAX_COLS - 1
    at = torch.arange(rows, device="cuda") * (wide // (rows - 1))  # from the first column to near the last
    at[-1] = wide - 1
    row = torch.arange(rows, device="cuda")
    assert cuts.gated(rows, wide, 8).sums.rows == cuts.gated(rows, 8, wide).dx.rows == 128
    x, w = torch.zeros(rows, wide, dtype=BF, device="cuda"), torch.ones(8, wide, dtype=BF, device="cuda")
    x[row, at] = (row + 1).to(BF)
    _, (g, u) = bk.rkb_gated_fwd(x, w, w, keep="full")
    assert torch.equal(g, (row + 1.0)[:, None].expand(rows, 8)) and torch.equal(u, g)
    del x, w
    dh = torch.zeros(rows, wide, dtype=BF, device="cuda")
    dh[row, at] = 1.0
    g, u = torch.zeros_like(dh), torch.full_like(dh, 2.0)  # silu(0) = 0 with a slope of 1/2: dg = dh, du = 0
    w = normal(torch.Generator(device="cuda").manual_seed(14), wide, 8, dtype=BF)
    x = torch.ones(rows, 8, dtype=BF, device="cuda")
    dx, dwg, dwu, _ = bk.rkb_gated_bwd(dh, x, w, w, kept=(g, u))
    assert torch.equal(dx, w[at])
    assert bool((dwg[at] == 1).all()) and int(dwg.count_nonzero()) == rows * 8 and not dwu.any()


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("cols", [100, 250, 500, 1000, 2000, 4000, 8000, 16384])
def test_layer_norm_columns_over_many_rows(cols, dtype):
    """dw and db over blocks that each take several rows in turn, the last turn not full, by every layout of a row."""
    rows, gen = 1403, torch.Generator(device="cuda").manual_seed(13)
    x, dy, w = normal(gen, rows, cols, dtype=dtype) + 0.5, normal(gen, rows, cols, dtype=dtype, scale=0.1), normal(gen, cols, dtype=dtype)
    _, mean, rstd = bk.rkb_layer_norm_fwd(x, w)
    c = bk.rkb_ckpt8_save(x)
    for kept, ref in ((x, x.double()), (c, bk.rkb_ckpt8_load(c).double())):
        args = (dy.double(), ref, mean.double(), rstd.double(), w.double())
        got = bk.rkb_layer_norm_bwd(dy, kept, mean, rstd, w, bias=True)
        for t, want, e in zip(got, bo.layer_norm_grads(*args), bo.layer_norm_grad_bounds(*args, dtype, dtype)):
            assert worst(t, want, e) <= 1.0
