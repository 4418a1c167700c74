"""The block operators (paper_2307_01236_amd/block.py) on an MI355X against their 64-bit definitions,
within the bounds that 32-bit sums and one rounding of each output allow (block_oracle)."""
import ctypes
import math

import pytest
import torch

import block_oracle as bo
from paper_2307_01236_amd import block as bk

pytestmark = pytest.mark.gpu
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def rand(*shape, seed=0, dtype=FP, scale=1.0, shift=0.0):
    t = torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale + shift
    return t.to(dtype).cuda()


def strided(t, extra=3, offset=1):
    """The same matrix as rows of a wider one, starting at an odd element."""
    wide = torch.full((t.shape[0], t.shape[1] + extra + offset), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, offset:offset + t.shape[1]] = t
    return wide[:, offset:offset + t.shape[1]]


# ------------------------------------------------------------------ layer norm

NORM_SHAPES = [(1, 1), (1, 1024), (3, 2), (5, 33), (17, 128), (64, 511), (777, 1001), (130, 1280), (33, 2048), (9, 2731),
               (7, 4096), (5, 8192), (3, 8200), (2, 16384), (1500, 64)]


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_layer_norm(rows, cols, dtype):
    eps = 1e-5
    x = rand(rows, cols, seed=1, dtype=dtype, shift=0.5)
    w, b = rand(cols, seed=2, dtype=dtype, shift=1.0), rand(cols, seed=3, dtype=dtype)
    y, mean, rstd = bk.rkb_layer_norm_fwd(x, w, b, eps)
    want = bo.layer_norm(bo.d(x), bo.d(w), bo.d(b), eps)
    bound = bo.layer_norm_bounds(bo.d(x), bo.d(w), bo.d(b), eps, dtype)
    for got, ref, e in zip((y, mean, rstd), want, bound):
        assert bo.worst(got, ref, e) <= 1.0
    dy = rand(rows, cols, seed=4, dtype=dtype, scale=0.1)
    dx, dw, db = bk.rkb_layer_norm_bwd(dy, x, mean, rstd, w, bias=True)
    args = (bo.d(dy), bo.d(x), bo.d(mean), bo.d(rstd), bo.d(w))
    for got, ref, e in zip((dx, dw, db), bo.layer_norm_grads(*args), bo.layer_norm_grad_bounds(*args, dtype, dtype)):
        assert bo.worst(got, ref, e) <= 1.0


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("rows,cols", [(1, 5), (40, 96), (333, 1000), (64, 1024), (5, 8192)])
def test_layer_norm_gradient_from_a_checkpoint(rows, cols, dtype):
    x, dy, w = (rand(rows, cols, seed=s, dtype=dtype) for s in (1, 2, 3))
    w = w[0].contiguous()
    _, mean, rstd = bk.rkb_layer_norm_fwd(x, w)
    c = bk.rkb_ckpt8_save(x)
    got = bk.rkb_layer_norm_bwd(dy, c, mean, rstd, w, bias=True)
    args = (bo.d(dy), bo.ckpt(bo.d(x), dtype)[2], bo.d(mean), bo.d(rstd), bo.d(w))
    for g, ref, e in zip(got, bo.layer_norm_grads(*args), bo.layer_norm_grad_bounds(*args, dtype, dtype)):
        assert bo.worst(g, ref, e) <= 1.0


def test_layer_norm_weights_of_other_type_or_none():
    x, dy = rand(50, 320, dtype=BF), rand(50, 320, seed=1, dtype=BF)
    w, b = rand(320, seed=2), rand(320, seed=3)  # 32-bit
    y, mean, rstd = bk.rkb_layer_norm_fwd(x, w, b)
    assert bo.worst(y, bo.layer_norm(bo.d(x), bo.d(w), bo.d(b), 1e-5)[0],
                    bo.layer_norm_bounds(bo.d(x), bo.d(w), bo.d(b), 1e-5, BF)[0]) <= 1.0
    dx, dw, db = bk.rkb_layer_norm_bwd(dy, x, mean, rstd, w, bias=True)
    assert dw.dtype == db.dtype == FP
    args = (bo.d(dy), bo.d(x), bo.d(mean), bo.d(rstd), bo.d(w))
    for g, ref, e in zip((dx, dw, db), bo.layer_norm_grads(*args), bo.layer_norm_grad_bounds(*args, BF, FP)):
        assert bo.worst(g, ref, e) <= 1.0
    y0, mean0, rstd0 = bk.rkb_layer_norm_fwd(x)
    assert torch.equal(mean0, mean) and torch.equal(rstd0, rstd)
    assert torch.equal(y0, bk.rkb_layer_norm_fwd(x, torch.ones(320, device="cuda"), torch.zeros(320, device="cuda"))[0])
    dx0, dw0, db0 = bk.rkb_layer_norm_bwd(dy, x, mean, rstd)
    assert dw0 is None and db0 is None
    args = (bo.d(dy), bo.d(x), bo.d(mean), bo.d(rstd), None)
    assert bo.worst(dx0, bo.layer_norm_grads(*args)[0], bo.layer_norm_grad_bounds(*args, BF, BF)[0]) <= 1.0
    assert torch.equal(bk.rkb_layer_norm_bwd(dy, x, mean, rstd, bias=True)[2].float(), db.to(BF).float())


def test_layer_norm_far_from_zero_and_flat_rows():
    """A mean a thousand deviations away, rows of one value, and a tiny scale."""
    x = rand(6, 1000, shift=1000.0)
    x[1] = 3.25
    x[2] = 0.0
    x[3] *= 1e-18
    y, mean, rstd = bk.rkb_layer_norm_fwd(x, eps=1e-5)
    want = bo.layer_norm(bo.d(x), None, None, 1e-5)
    for got, ref, e in zip((y, mean, rstd), want, bo.layer_norm_bounds(bo.d(x), None, None, 1e-5, FP)):
        assert bo.worst(got, ref, e) <= 1.0
    assert bool((y[1:3] == 0).all()) and math.isclose(float(rstd[2]), 1e-5 ** -0.5, rel_tol=1e-6)


def test_layer_norm_with_pointers_left_out():
    """At the C interface: no statistics, a bias without a weight, one of dw and db alone."""
    lib, st = bk.load(), torch.cuda.current_stream().cuda_stream
    x, dy, b = rand(70, 130, dtype=HF), rand(70, 130, seed=1, dtype=HF), rand(130, seed=2, dtype=HF)
    want, mean, rstd = bk.rkb_layer_norm_fwd(x, None, b)
    y = torch.empty_like(x)
    assert lib.rkb_layer_norm_fwd(bk.RKB_F16, bk.RKB_F16, 70, 130, x.data_ptr(), 130, None, b.data_ptr(), 1e-5, y.data_ptr(), 130,
                                  None, None, st) == 0
    assert torch.equal(y, want)
    _, dw, db = bk.rkb_layer_norm_bwd(dy, x, mean, rstd, torch.ones_like(b), bias=True)
    n = ctypes.c_size_t(0)
    assert lib.rkb_layer_norm_bwd_workspace(bk.RKB_F16, 70, 130, ctypes.byref(n)) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    for which in (0, 1):
        out = [torch.zeros_like(b), torch.zeros_like(b)]
        ptrs = [None, None]
        ptrs[which] = out[which].data_ptr()
        assert lib.rkb_layer_norm_bwd(bk.RKB_F16, bk.RKB_F16, 70, 130, dy.data_ptr(), 130, x.data_ptr(), 130, None, None,
                                      mean.data_ptr(), rstd.data_ptr(), None, y.data_ptr(), 130, *ptrs, ws.data_ptr(), n.value,
                                      st) == 0
        assert torch.equal(out[which], (dw, db)[which]) and not out[1 - which].any()


def test_layer_norm_keeps_a_bad_row_to_itself():
    x, dy, w = rand(9, 300, dtype=HF), rand(9, 300, seed=1, dtype=HF), rand(300, seed=2, dtype=HF)
    clean = bk.rkb_layer_norm_fwd(x, w)
    x[4, 7], x[6, 299] = float("nan"), float("inf")
    y, mean, rstd = bk.rkb_layer_norm_fwd(x, w)
    good = [0, 1, 2, 3, 5, 7, 8]
    assert bool(y[4].isnan().all()) and bool(y[6].isnan().all())
    assert all(torch.equal(a[good], b[good]) for a, b in zip((y, mean, rstd), clean))
    dx = bk.rkb_layer_norm_bwd(dy, x, mean, rstd, w)[0]
    assert bool(dx[good].isfinite().all()) and bool(dx[4].isnan().all())


def test_layer_norm_rows_apart_and_leading_dimensions():
    x, dy, w = rand(60, 200, dtype=BF), rand(60, 200, seed=1, dtype=BF), rand(200, seed=2, dtype=BF)
    want = bk.rkb_layer_norm_fwd(x, w)
    got = bk.rkb_layer_norm_fwd(strided(x), w)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    cube = bk.rkb_layer_norm_fwd(x.view(3, 20, 200), w)
    assert cube[0].shape == (3, 20, 200) and cube[1].shape == (3, 20) and torch.equal(cube[0].view(60, 200), want[0])
    _, mean, rstd = want
    a = bk.rkb_layer_norm_bwd(dy, x, mean, rstd, w, bias=True)
    b = bk.rkb_layer_norm_bwd(strided(dy, 8, 3), strided(x, 1, 2), mean, rstd, w, bias=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_layer_norm_gradient_is_the_difference():
    """A 32-bit forward's change along a direction against the gradient: the sum over many outputs of
    roundings of u * |y dy| each, over a step of 1/64."""
    rows, cols, h = 16, 300, 1 / 64
    x, w, b, dy = rand(rows, cols), rand(cols, seed=1), rand(cols, seed=2), rand(rows, cols, seed=3)
    _, mean, rstd = bk.rkb_layer_norm_fwd(x, w, b)
    grads = bk.rkb_layer_norm_bwd(dy, x, mean, rstd, w, bias=True)
    for i, at in enumerate((x, w, b)):
        v = rand(*at.shape, seed=7 + i)
        v /= v.norm()
        plus, minus = [x, w, b], [x, w, b]
        plus[i], minus[i] = at + h * v, at - h * v
        loss = [float((bo.d(bk.rkb_layer_norm_fwd(*t)[0]) * bo.d(dy)).sum()) for t in (plus, minus)]
        rounding = 8 * bo.U32 * float((bo.d(bk.rkb_layer_norm_fwd(x, w, b)[0]) * bo.d(dy)).abs().sum()) / h
        curve = h * h * float(dy.norm()) * 8  # third derivatives along a unit direction, generously
        assert abs((loss[0] - loss[1]) / (2 * h) - float((bo.d(grads[i]) * bo.d(v)).sum())) <= rounding + curve


# ------------------------------------------------------------------ checkpoints

@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (70, 64), (1031, 2731), (19, 4096), (2, 8193),
                                       (300, 100), (4000, 48)])
def test_checkpoint(rows, cols, dtype):
    x = rand(rows, cols, dtype=dtype) * torch.exp(rand(rows, 1, seed=1)).to(dtype)
    x[0, :1] = 0
    c = bk.rkb_ckpt8_save(x)
    q, e, v = bo.ckpt(bo.d(x), dtype)
    assert torch.equal(bo.d(c.codes)[:, :cols], q) and bool((c.codes[:, cols:] == 0).all())
    assert torch.equal(c.exps.cpu().double(), e + 127)
    got = bk.rkb_ckpt8_load(c)
    assert got.dtype == dtype and got.shape == x.shape and torch.equal(bo.d(got), v)
    assert c.nbytes() == rows * -(-cols // 32) * 33


@pytest.mark.parametrize("dtype", [BF, HF, FP])
def test_checkpoint_at_the_ends_of_the_range(dtype):
    info = torch.finfo(dtype)
    tiny = 2.0 ** -24 if dtype == HF else 2.0 ** -133  # a subnormal of the type
    x = torch.zeros(8, 64, dtype=dtype, device="cuda")
    x[0] = info.max
    x[1] = -info.max
    x[2, ::2] = info.max
    x[2, 1::2] = info.max / 130
    x[3] = info.tiny
    x[4, 5] = tiny
    x[5, :32] = torch.arange(32, device="cuda") * tiny
    x[6, 3] = -0.0
    x[7] = 127.5 * 2.0 ** -3  # a tie at the code's limit
    c = bk.rkb_ckpt8_save(x)
    q, e, v = bo.ckpt(bo.d(x), dtype)
    assert torch.equal(bo.d(c.codes), q) and torch.equal(c.exps.cpu().double(), e + 127)
    assert torch.equal(bo.d(bk.rkb_ckpt8_load(c)), v)


def test_checkpoint_of_infinities_and_nan():
    x = rand(4, 96, dtype=BF)
    x[0, 3], x[1, 40], x[3, 95] = float("inf"), float("nan"), -float("inf")
    bad = torch.zeros(4, 3, dtype=torch.bool, device="cuda")
    bad[0, 0] = bad[1, 1] = bad[3, 2] = True
    got = bk.rkb_ckpt8_load(bk.rkb_ckpt8_save(x)).view(4, 3, 32)
    assert bool(got[bad].isnan().all()) and bool(got[~bad].isfinite().all())
    clean = bo.ckpt(bo.d(torch.where(bad.repeat_interleave(32, 1), 0, x)), BF)[2].view(4, 3, 32)
    assert torch.equal(bo.d(got[~bad]), clean[~bad.cpu()])


def test_checkpoint_of_rows_apart_and_leading_dimensions():
    x = rand(40, 70, dtype=HF)
    want = bk.rkb_ckpt8_save(x)
    got = bk.rkb_ckpt8_save(strided(x))
    assert torch.equal(want.codes, got.codes) and torch.equal(want.exps, got.exps)
    assert bk.rkb_ckpt8_load(bk.rkb_ckpt8_save(x.view(5, 8, 70))).shape == (5, 8, 70)


# ------------------------------------------------------------------ products

WGRAD_SHAPES = [(1, 1, 1), (1, 64, 64), (2, 33, 65), (37, 100, 40), (64, 128, 256), (129, 257, 130), (500, 72, 1000),
                (1031, 90, 333), (256, 512, 512), (2048, 264, 384), (4100, 24, 40)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("form", ["ckpt", "full"])
@pytest.mark.parametrize("rows,n,k", WGRAD_SHAPES)
def test_weight_grad(rows, n, k, form, dtype):
    dy, x = rand(rows, n, dtype=dtype), rand(rows, k, seed=1, dtype=dtype)
    kept = bo.ckpt(bo.d(x), dtype)[2] if form == "ckpt" else bo.d(x)
    got = bk.rkb_weight_grad(dy, bk.rkb_ckpt8_save(x) if form == "ckpt" else x)
    ref = bo.d(dy).t() @ kept
    bound = bo.sum_bound(bo.d(dy).abs().t() @ kept.abs(), rows) + bo.rounding(ref, dtype)
    assert bo.worst(got, ref, bound) <= 1.0


@pytest.mark.parametrize("rows,n,k", [(1024, 22528, 4096), (1024, 22533, 4096)])
def test_weight_grad_of_many_tiles(rows, n, k):
    """Several rounds of large tiles, the last one part empty; element by element."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    dy, x = (torch.randn(rows, c, generator=gen, device="cuda").to(BF) for c in (n, k))
    got = bk.rkb_weight_grad(dy, x)
    for at in range(0, n, 4096):  # rows of dw, a few at a time in 64 bits
        ref = torch.mm(dy[:, at:at + 4096].t().double().contiguous(), x.double())
        bound = (rows + 8) * bo.U32 * torch.mm(dy[:, at:at + 4096].t().abs().double().contiguous(), x.abs().double()) \
            + ref.abs() * bo.ROUND[BF][0]
        assert float(((got[at:at + 4096].double() - ref).abs() / bound).max()) <= 1.0


def test_weight_grad_of_rows_apart():
    dy, x = rand(300, 72, dtype=BF), rand(300, 136, seed=1, dtype=BF)
    want = bk.rkb_weight_grad(dy, x)
    assert torch.equal(bk.rkb_weight_grad(strided(dy), strided(x)), want)
    assert torch.equal(bk.rkb_weight_grad(strided(dy, 16, 0), strided(x, 7, 8)), want)


GATED_SHAPES = [(1, 1, 1), (1, 64, 96), (1, 1024, 512), (2, 40, 33), (3, 1000, 130), (8, 33, 40), (16, 72, 2730), (17, 256, 64),
                (37, 1000, 274), (64, 64, 64), (65, 129, 257), (130, 512, 200), (257, 320, 264), (513, 136, 1100)]


def gated_inputs(rows, width, hidden, dtype):
    x = rand(rows, width, seed=1, dtype=dtype)
    wg, wu = (rand(hidden, width, seed=s, dtype=dtype, scale=width ** -0.5) for s in (2, 3))
    return x, wg, wu, rand(rows, hidden, seed=4, dtype=dtype, scale=0.1)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,width,hidden", GATED_SHAPES)
def test_gated(rows, width, hidden, act, dtype):
    x, wg, wu, dh = gated_inputs(rows, width, hidden, dtype)
    X, G, U, DH = bo.d(x), bo.d(wg), bo.d(wu), bo.d(dh)
    h_ref, g_ref, u_ref = bo.gated(X, G, U, act)
    h_bound, eg, eu = bo.gated_bounds(X, G, U, act, dtype)
    first = None
    for keep in ("none", "full", "16bit", "8bit"):
        h, kept = bk.rkb_gated_fwd(x, wg, wu, act, keep=keep)
        assert h.shape == (rows, hidden) and bo.worst(h, h_ref, h_bound) <= 1.0, keep
        if first is not None:
            assert torch.equal(h, first)  # the same h whatever is kept
        first = h
        if keep == "none":
            assert kept is None
            g, u, slack = g_ref, u_ref, (eg, eu)
        elif keep in ("full", "16bit"):
            kind = FP if keep == "full" else dtype
            for t, ref, e in zip(kept, (g_ref, u_ref), (eg, eu)):
                assert t.dtype == kind and bo.worst(t, ref, e + bo.rounding(ref, kind) * 1.01) <= 1.0
            g, u, slack = bo.d(kept[0]), bo.d(kept[1]), (0.0, 0.0)
        else:
            vals = []
            for c, ref, e in zip(kept, (g_ref, u_ref), (eg, eu)):
                step = torch.exp2(c.exps.cpu().double() - 127).repeat_interleave(32, 1)
                assert bool((c.codes[:, hidden:] == 0).all())
                vals.append((bo.d(c.codes) * step)[:, :hidden])
                assert bo.worst(vals[-1], ref, step[:, :hidden] / 2 + 2 * e) <= 1.0
                top = torch.exp2(bo.ckpt_step(ref)) + 127  # at most one step off where the maximum is at a boundary
                assert bool(((c.exps.cpu().double() - 127 - bo.ckpt_step(ref)).abs() <= 1).all()) and top.numel()
            (g, u), slack = vals, (0.0, 0.0)
        got = bk.rkb_gated_bwd(dh, x, wg, wu, act, kept, want_h=True)
        refs = bo.gated_grads(DH, X, G, U, act, g, u)
        for name, t, ref, e in zip(("dx", "dwg", "dwu", "h"), got, refs,
                                   bo.gated_grad_bounds(DH, X, G, U, act, g, u, dtype, *slack)):
            assert bo.worst(t, ref, e) <= 1.0, (keep, name)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,width,hidden", [(1, 1, 1), (1, 64, 64), (3, 1000, 130), (40, 24, 96), (1, 96, 4096)])
def test_gated_gradients_of_few_elements_round_once(rows, width, hidden, dtype):
    """Up to 4096 elements of dg enter the products in two parts, so that only the results are rounded."""
    x, wg, wu, dh = gated_inputs(rows, width, hidden, dtype)
    args = (bo.d(dh), bo.d(x), bo.d(wg), bo.d(wu), "silu")
    kept = bk.rkb_gated_fwd(x, wg, wu, keep="full")[1]
    g, u = bo.d(kept[0]), bo.d(kept[1])
    got = bk.rkb_gated_bwd(dh, x, wg, wu, kept=kept)
    for t, ref, e in zip(got[:3], bo.gated_grads(*args, g, u), bo.gated_grad_bounds(*args, g, u, dtype, fine=True)):
        assert bo.worst(t, ref, e) <= 1.0
    assert all(torch.equal(p, q) for p, q in zip(got[:3], bk.rkb_gated_bwd(dh, x, wg, wu)[:3]))


def test_gated_one_gradient_alone():
    """dx or the weights' gradients left out at the C interface: the others are the same."""
    lib = bk.load()
    for rows, width, hidden in ((3, 64, 96), (300, 136, 264), (1500, 72, 520)):
        x, wg, wu, dh = gated_inputs(rows, width, hidden, BF)
        kept = bk.rkb_gated_fwd(x, wg, wu, keep="16bit")[1]
        want = bk.rkb_gated_bwd(dh, x, wg, wu, kept=kept)
        n = ctypes.c_size_t(0)
        assert lib.rkb_gated_bwd_workspace(bk.RKB_BF16, bk.RKB_KEEP_16BIT, rows, width, hidden, 1, ctypes.byref(n)) == 0
        ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
        for only_dx in (True, False):
            dx, dwg, dwu = (torch.zeros_like(t) for t in want[:3])
            rc = lib.rkb_gated_bwd(bk.RKB_BF16, bk.RKB_SILU, bk.RKB_KEEP_16BIT, rows, width, hidden, dh.data_ptr(), hidden,
                                   x.data_ptr(), width, wg.data_ptr(), width, wu.data_ptr(), width, kept[0].data_ptr(),
                                   kept[1].data_ptr(), None, None, dx.data_ptr() if only_dx else None, width,
                                   None if only_dx else dwg.data_ptr(), None if only_dx else dwu.data_ptr(), width, None, hidden,
                                   ws.data_ptr(), n.value, torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            close = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm()) <= bo.ROUND[BF][0]  # noqa: E731
            # by another cut of the sum the last bit may differ
            assert close(dx, want[0]) if only_dx else close(dwg, want[1]) and close(dwu, want[2])


def test_gated_far_ends_of_the_activation():
    """Gates from -100 to 100: nothing overflows, and far below zero h and the gradients vanish."""
    for act in ("silu", "gelu"):
        x = torch.linspace(-100, 100, 64, device="cuda").to(BF).view(64, 1)
        wg, wu = torch.ones(3, 1, device="cuda", dtype=BF), torch.full((3, 1), 0.5, device="cuda", dtype=BF)
        dh = torch.ones(64, 3, device="cuda", dtype=BF)
        h_ref, g, u = bo.gated(bo.d(x), bo.d(wg), bo.d(wu), act)
        bound, eg, eu = bo.gated_bounds(bo.d(x), bo.d(wg), bo.d(wu), act, BF)
        for keep in ("none", "full"):
            h, kept = bk.rkb_gated_fwd(x, wg, wu, act, keep=keep)
            assert bo.worst(h, h_ref, bound) <= 1.0
            got = bk.rkb_gated_bwd(dh, x, wg, wu, act, kept)
            args = (bo.d(dh), bo.d(x), bo.d(wg), bo.d(wu), act, g, u)
            for t, ref, e in zip(got[:3], bo.gated_grads(*args)[:3], bo.gated_grad_bounds(*args, BF, eg, eu)):
                assert bo.worst(t, ref, e) <= 1.0


def test_gated_rows_apart_and_leading_dimensions():
    x, wg, wu, dh = gated_inputs(66, 136, 200, BF)
    for keep in ("none", "full", "16bit", "8bit"):
        h, kept = bk.rkb_gated_fwd(x, wg, wu, keep=keep)
        want = bk.rkb_gated_bwd(dh, x, wg, wu, kept=kept)
        h2, kept2 = bk.rkb_gated_fwd(strided(x), strided(wg, 8, 0), strided(wu, 2, 1), keep=keep)
        got = bk.rkb_gated_bwd(strided(dh), strided(x, 8, 8), strided(wg, 1, 0), strided(wu), kept=kept2)
        assert torch.equal(h, h2) and all(torch.equal(a, b) for a, b in zip(want[:3], got[:3]))
    h3, kept3 = bk.rkb_gated_fwd(x.view(3, 22, 136), wg, wu, keep="8bit")
    assert h3.shape == (3, 22, 200) and torch.equal(h3.view(66, 200), h)
    dx = bk.rkb_gated_bwd(dh.view(3, 22, 200), x.view(3, 22, 136), wg, wu, kept=kept3)[0]
    assert dx.shape == (3, 22, 136) and torch.equal(dx.view(66, 136), want[0])


def test_gated_keeps_a_bad_token_to_itself():
    x, wg, wu, dh = gated_inputs(70, 136, 200, BF)
    clean_h, kept = bk.rkb_gated_fwd(x, wg, wu, keep="8bit")
    clean_dx = bk.rkb_gated_bwd(dh, x, wg, wu, kept=kept)[0]
    x[5, 3] = float("nan")
    h, kept = bk.rkb_gated_fwd(x, wg, wu, keep="8bit")
    got = bk.rkb_gated_bwd(dh, x, wg, wu, kept=kept)
    others = [i for i in range(70) if i != 5]
    assert bool(h[5].isnan().all()) and torch.equal(h[others], clean_h[others])
    assert bool(got[0][5].isnan().all()) and torch.equal(got[0][others], clean_dx[others])
    assert bool(got[1].isnan().all())  # every weight saw the token


@pytest.mark.parametrize("act,dtype", [("silu", BF), ("gelu", HF)])
@pytest.mark.parametrize("rows,width,hidden", [(1000, 520, 8200), (4100, 72, 3000), (3000, 264, 2056), (4096, 4096, 72),
                                               (40, 2000, 6000), (90, 4096, 2000)])
def test_gated_at_sizes_of_every_tile(rows, width, hidden, act, dtype):
    """Large enough for the larger tiles, split sums and many workgroups; the 64-bit side runs on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, wg, wu, dh = (torch.randn(*s, generator=gen, device="cuda").mul_(f).to(dtype) for s, f in (
        ((rows, width), 1.0), ((hidden, width), width ** -0.5), ((hidden, width), width ** -0.5), ((rows, hidden), 0.1)))
    X, G, U, DH = x.double(), wg.double(), wu.double(), dh.double()
    mm = lambda a, b: torch.mm(a.contiguous(), b.contiguous())  # noqa: E731
    g, u = mm(X, G.t()), mm(X, U.t())
    a, s = bo.act(g, act)
    h, kept = bk.rkb_gated_fwd(x, wg, wu, act, keep="full")
    assert float(((h.double() - a * u).norm() / (a * u).norm())) <= bo.ROUND[dtype][0]
    for t, ref in zip(kept, (g, u)):
        assert float((t.double() - ref).abs().max()) <= bo.U32 * width * float(mm(X.abs(), G.abs().t()).max())
    dx, dwg, dwu, h2 = bk.rkb_gated_bwd(dh, x, wg, wu, act, kept, want_h=True)
    again = bk.rkb_gated_bwd(dh, x, wg, wu, act, None, want_h=True)
    assert torch.equal(h, h2) and all(torch.equal(p, q) for p, q in zip((dx, dwg, dwu, h2), again))
    dg, du = DH * u * s, DH * a
    # each operand dg or du and each output is rounded once: two roundings of u, rms below the bound of one
    for got, ref in ((dx, mm(dg, G) + mm(du, U)), (dwg, mm(dg.t(), X)), (dwu, mm(du.t(), X))):
        assert float((got.double() - ref).norm() / ref.norm()) <= bo.ROUND[dtype][0]


def test_offsets_past_32_bits():
    """Rows 2^22 elements apart, and matrices of more than 2^31 elements."""
    far = 1 << 22
    store = torch.zeros(1100 * far // 2, dtype=BF, device="cuda")  # 2.3e9 elements
    x = torch.as_strided(store, (540, 64), (far, 1))
    x.copy_(rand(540, 64, seed=1, dtype=BF))
    near = x.clone()
    wg, wu, dh = rand(96, 64, seed=2, dtype=BF), rand(96, 64, seed=3, dtype=BF), rand(540, 96, seed=4, dtype=BF)
    a, b = bk.rkb_gated_fwd(x, wg, wu, keep="8bit"), bk.rkb_gated_fwd(near, wg, wu, keep="8bit")
    assert torch.equal(a[0], b[0])
    assert all(torch.equal(p, q) for p, q in zip(bk.rkb_gated_bwd(dh, x, wg, wu, kept=a[1])[:3],
                                                 bk.rkb_gated_bwd(dh, near, wg, wu, kept=b[1])[:3]))
    assert torch.equal(bk.rkb_weight_grad(dh, x), bk.rkb_weight_grad(dh, near))
    assert all(torch.equal(p, q) for p, q in zip(bk.rkb_layer_norm_fwd(x), bk.rkb_layer_norm_fwd(near)))
    assert torch.equal(bk.rkb_ckpt8_save(x).codes, bk.rkb_ckpt8_save(near).codes)
    del store, x
    rows, cols = (1 << 18) + 3, 8200
    big = torch.empty(rows, cols, dtype=BF, device="cuda").normal_()
    y, mean, rstd = bk.rkb_layer_norm_fwd(big)
    c = bk.rkb_ckpt8_save(big)
    dx = bk.rkb_layer_norm_bwd(big, c, mean, rstd)[0]
    values = bk.rkb_ckpt8_load(c)
    last = big[-5:].clone()
    y2, mean2, rstd2 = bk.rkb_layer_norm_fwd(last)
    c2 = bk.rkb_ckpt8_save(last)
    assert torch.equal(y[-5:], y2) and torch.equal(mean[-5:], mean2) and torch.equal(rstd[-5:], rstd2)
    assert torch.equal(c.codes[-5:], c2.codes) and torch.equal(values[-5:], bk.rkb_ckpt8_load(c2))
    assert torch.equal(dx[-5:], bk.rkb_layer_norm_bwd(last, c2, mean2, rstd2)[0])


def test_broadcast_rows():
    """One row that stands for all of an input (a stride of 0), as an expanded gradient has."""
    x, wg, wu, _ = gated_inputs(70, 136, 200, BF)
    dy, dh = rand(1, 136, seed=8, dtype=BF), rand(1, 200, seed=9, dtype=BF)
    _, mean, rstd = bk.rkb_layer_norm_fwd(x)
    wide, full = dy.expand(70, 136), dy.expand(70, 136).contiguous()
    for p, q in zip(bk.rkb_layer_norm_bwd(wide, x, mean, rstd, bias=True), bk.rkb_layer_norm_bwd(full, x, mean, rstd, bias=True)):
        assert (p is None and q is None) or torch.equal(p, q)
    assert torch.equal(bk.rkb_weight_grad(wide, x), bk.rkb_weight_grad(full, x))
    for kept in (None, bk.rkb_gated_fwd(x, wg, wu, keep="8bit")[1]):
        assert all(torch.equal(p, q) for p, q in zip(bk.rkb_gated_bwd(dh.expand(70, 200), x, wg, wu, kept=kept)[:3],
                                                     bk.rkb_gated_bwd(dh.expand(70, 200).contiguous(), x, wg, wu, kept=kept)[:3]))
    assert torch.equal(bk.rkb_ckpt8_save(wide).codes, bk.rkb_ckpt8_save(full).codes)


# ------------------------------------------------------------------ calls

def all_calls(x, w, b, dy, wg, wu, dh):
    y, mean, rstd = bk.rkb_layer_norm_fwd(x, w, b)
    c = bk.rkb_ckpt8_save(x)
    out = [y, mean, rstd, bk.rkb_ckpt8_load(c), bk.rkb_weight_grad(dy, c)]
    out += bk.rkb_layer_norm_bwd(dy, c, mean, rstd, w, bias=True)
    for keep in ("none", "full", "16bit", "8bit"):
        h, kept = bk.rkb_gated_fwd(y, wg, wu, keep=keep)
        out.append(h)
        out += bk.rkb_gated_bwd(dh, y, wg, wu, kept=kept, want_h=True)
    return out


def call_inputs(rows=300, width=264, hidden=520):
    x, wg, wu, dh = gated_inputs(rows, width, hidden, BF)
    return x, rand(width, seed=5, dtype=BF), rand(width, seed=6, dtype=BF), rand(rows, width, seed=7, dtype=BF), wg, wu, dh


def test_results_repeat_bit_for_bit():
    args = call_inputs()
    a, b = all_calls(*args), all_calls(*args)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_another_stream():
    args = call_inputs()
    want = all_calls(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy = torch.zeros(1 << 26, device="cuda")
        for _ in range(20):
            busy += 1  # the calls must come after this on the side stream, not beside it
        late = args[0] + (busy[0] - 20).to(BF)
        got = all_calls(late, *args[1:])
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_graph_replays():
    """Captured once, replayed over changed inputs with eager work between."""
    args = call_inputs(130, 136, 200)
    static = [t.clone() for t in args]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_calls(*static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = all_calls(*static)
    for rep in range(4):
        for s, t in zip(static, args):
            s.copy_(t * (1.0 + rep))
        graph.replay()
        torch.cuda.synchronize()
        want = all_calls(*static)
        assert all(torch.equal(p, q) for p, q in zip(want, out)), rep


def test_no_rows():
    x, w = torch.zeros(0, 64, dtype=BF, device="cuda"), rand(40, 64, dtype=BF)
    y, mean, rstd = bk.rkb_layer_norm_fwd(x)
    assert y.shape == (0, 64) and mean.shape == rstd.shape == (0,)
    dx, dw, db = bk.rkb_layer_norm_bwd(x, x, mean, rstd, w[0], bias=True)
    assert dx.shape == (0, 64) and bool((dw == 0).all()) and bool((db == 0).all())
    c = bk.rkb_ckpt8_save(x)
    assert bk.rkb_ckpt8_load(c).shape == (0, 64)
    assert bool((bk.rkb_weight_grad(torch.zeros(0, 40, dtype=BF, device="cuda"), c) == 0).all())
    for keep in ("none", "full", "16bit", "8bit"):
        h, kept = bk.rkb_gated_fwd(x, w, w, keep=keep)
        assert h.shape == (0, 40)
        dx, dwg, dwu, _ = bk.rkb_gated_bwd(h, x, w, w, kept=kept)
        assert dx.shape == (0, 64) and bool((dwg == 0).all()) and bool((dwu == 0).all())


def test_the_binding_refuses_what_does_not_fit():
    x, wg, wu, dh = gated_inputs(8, 64, 40, BF)
    c = bk.rkb_ckpt8_save(x)
    y, mean, rstd = bk.rkb_layer_norm_fwd(x)
    bad = [
        lambda: bk.rkb_layer_norm_fwd(x.t()),
        lambda: bk.rkb_layer_norm_fwd(x, wg[0].half()),
        lambda: bk.rkb_layer_norm_fwd(x, wg[0, :63]),
        lambda: bk.rkb_layer_norm_fwd(x, wg[0], wu[0].float()),
        lambda: bk.rkb_layer_norm_fwd(torch.zeros(2, 16385, dtype=BF, device="cuda")),
        lambda: bk.rkb_layer_norm_bwd(x, x[:7], mean, rstd),
        lambda: bk.rkb_layer_norm_bwd(x, x.half(), mean, rstd),
        lambda: bk.rkb_layer_norm_bwd(x, x, mean[:7], rstd),
        lambda: bk.rkb_layer_norm_bwd(x, x, mean.half(), rstd),
        lambda: bk.rkb_layer_norm_bwd(x.half(), c, mean, rstd),
        lambda: bk.rkb_layer_norm_bwd(x[:7], c, mean[:7], rstd[:7]),
        lambda: bk.rkb_ckpt8_save(x.double()),
        lambda: bk.rkb_ckpt8_save(x.view(8, 8, 8).transpose(0, 1)),
        lambda: bk.rkb_ckpt8_load(x),
        lambda: bk.rkb_ckpt8_load(bk.Ckpt8(c.codes[:7], c.exps, c.shape, c.dtype)),
        lambda: bk.rkb_weight_grad(x[:7], c),
        lambda: bk.rkb_weight_grad(x.float(), x.float()),
        lambda: bk.rkb_gated_fwd(x, wg, wu[:39]),
        lambda: bk.rkb_gated_fwd(x, wg[:, :63], wu),
        lambda: bk.rkb_gated_fwd(x, wg.half(), wu),
        lambda: bk.rkb_gated_bwd(dh[:7], x, wg, wu),
        lambda: bk.rkb_gated_bwd(dh, x, wg, wu, kept=(dh, dh[:7])),
        lambda: bk.rkb_gated_bwd(dh, x, wg, wu, kept=(dh, strided(dh))),
        lambda: bk.rkb_gated_bwd(dh, x, wg, wu, kept=(dh, dh.float())),
        lambda: bk.rkb_gated_bwd(dh, x, wg, wu, kept=(dh.half(), dh.half())),
        lambda: bk.rkb_gated_bwd(dh, x, wg, wu, kept=(bk.rkb_ckpt8_save(dh),) * 2),  # of a 16-bit type
    ]
    for i, call in enumerate(bad):
        with pytest.raises(bk.RKBError) as e:
            call()
        assert e.value.code == bk.RKB_E_INVAL, i


@pytest.mark.parametrize("rows,hidden", [(3, 40), (70, 72)])
def test_gated_gradients_past_the_range(rows, hidden):
    """dg or du beyond the largest value of 16 bits: the infinity that it rounds to reaches the gradients it belongs to, and no
    other, with its sign, for few elements (two parts) as for many."""
    width, at = 24, (1, 5)
    x, wg, wu = (torch.full(s, 0.5, dtype=HF, device="cuda") for s in ((rows, width), (hidden, width), (hidden, width)))
    for which in ("g", "u"):
        for sign in (1.0, -1.0):
            g, u = (torch.ones(rows, hidden, device="cuda") for _ in range(2))
            (u if which == "g" else g)[at] = 1000.0  # dg = dh u act'(g), du = dh act(g)
            dh = torch.full((rows, hidden), 0.01, dtype=HF, device="cuda")
            dh[at] = 200.0 * sign
            dx, dwg, dwu, _ = bk.rkb_gated_bwd(dh, x, wg, wu, kept=(g, u))
            bad, good = (dwg, dwu) if which == "g" else (dwu, dwg)
            assert bool((dx[at[0]] == sign * math.inf).all()) and bool((bad[at[1]] == sign * math.inf).all())
            assert bool(good.isfinite().all())
            others = torch.arange(rows, device="cuda") != at[0], torch.arange(hidden, device="cuda") != at[1]
            assert bool(dx[others[0]].isfinite().all()) and bool(bad[others[1]].isfinite().all())


@pytest.mark.parametrize("rows,hidden", [(3, 40), (70, 72)])
def test_gated_gradients_of_a_bad_element(rows, hidden):
    """NaN and infinities in dh stay NaN and infinities where they belong."""
    x, wg, wu = (torch.full(s, 0.5, dtype=BF, device="cuda") for s in ((rows, 24), (hidden, 24), (hidden, 24)))
    one = torch.ones(rows, hidden, device="cuda")
    for value, check in ((math.nan, torch.isnan), (math.inf, torch.isposinf), (-math.inf, torch.isneginf)):
        dh = torch.full((rows, hidden), 0.01, dtype=BF, device="cuda")
        dh[2, 7] = value
        dx, dwg, dwu, _ = bk.rkb_gated_bwd(dh, x, wg, wu, kept=(one, one))
        for t, line in ((dx, 2), (dwg, 7), (dwu, 7)):
            assert bool(check(t[line]).all()) and int(t.isfinite().all(1).sum()) == t.shape[0] - 1


@pytest.mark.parametrize("lead", [(3, 0), (0, 3), (0, 3, 5), (2, 0, 5), (0,)])
def test_no_rows_of_any_leading_dimensions(lead):
    x, dh, w = torch.zeros(*lead, 64, dtype=BF, device="cuda"), torch.zeros(*lead, 40, dtype=BF, device="cuda"), rand(40, 64, dtype=BF)
    y, mean, rstd = bk.rkb_layer_norm_fwd(x)
    assert y.shape == x.shape and mean.shape == lead
    dx, _, db = bk.rkb_layer_norm_bwd(x, x, mean, rstd, bias=True)
    assert dx.shape == x.shape and not db.any()
    c = bk.rkb_ckpt8_save(x)
    assert bk.rkb_ckpt8_load(c).shape == x.shape
    assert not bk.rkb_weight_grad(dh, c).any() and not bk.rkb_weight_grad(dh, x).any()
    for keep in ("none", "full", "16bit", "8bit"):
        h, kept = bk.rkb_gated_fwd(x, w, w, keep=keep)
        assert h.shape == dh.shape
        dx, dwg, dwu, again = bk.rkb_gated_bwd(dh, x, w, w, kept=kept, want_h=True)
        assert dx.shape == x.shape and again.shape == dh.shape and not dwg.any() and not dwu.any()
    wide = torch.zeros(*lead, 80, dtype=BF, device="cuda")[..., 3:67]  # no elements, whatever the strides
    assert bk.rkb_layer_norm_fwd(wide)[0].shape == x.shape and bk.rkb_ckpt8_save(wide).shape == x.shape


def test_an_earlier_error_is_neither_reported_nor_cleared():
    """An error that some call before left with the HIP runtime is not these calls', and stays for whoever asks for it.  At
    the C interface: torch's allocator asks by itself."""
    rows, d, f = 100, 64, 96
    lib, st = bk.load(), torch.cuda.current_stream().cuda_stream
    x, wg, wu, dh = gated_inputs(rows, d, f, BF)
    y, dx, h, dw, dwg, dwu = (torch.zeros(s, dtype=BF, device="cuda") for s in ((rows, d), (rows, d), (rows, f), (f, d), (f, d), (f, d)))
    mean, rstd = (torch.zeros(rows, device="cuda") for _ in range(2))
    codes, exps = torch.zeros(rows, d, dtype=torch.int8, device="cuda"), torch.zeros(rows, d // 32, dtype=torch.uint8, device="cuda")
    db = torch.zeros(d, dtype=BF, device="cuda")
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    p, B = (lambda t: t.data_ptr()), bk.RKB_BF16
    calls = [
        lambda: lib.rkb_layer_norm_fwd(B, B, rows, d, p(x), d, None, None, 1e-5, p(y), d, p(mean), p(rstd), st),
        lambda: lib.rkb_ckpt8_save(B, rows, d, p(x), d, p(codes), p(exps), st),
        lambda: lib.rkb_ckpt8_load(B, rows, d, p(codes), p(exps), p(y), d, st),
        lambda: lib.rkb_weight_grad(B, rows, f, d, p(dh), f, None, d, p(codes), p(exps), p(dw), d, p(ws), 1 << 24, st),
        lambda: lib.rkb_layer_norm_bwd(B, B, rows, d, p(x), d, p(x), d, None, None, p(mean), p(rstd), None, p(dx), d, None, p(db), p(ws),
                                       1 << 24, st),
        lambda: lib.rkb_gated_fwd(B, 0, 0, rows, d, f, p(x), d, p(wg), d, p(wu), d, p(h), f, None, None, None, None, p(ws), 1 << 24, st),
        lambda: lib.rkb_gated_bwd(B, 0, 0, rows, d, f, p(dh), f, p(x), d, p(wg), d, p(wu), d, None, None, None, None, p(dx), d, p(dwg),
                                  p(dwu), d, None, f, p(ws), 1 << 24, st),
    ]
    torch.cuda.synchronize()
    lib.hipGetLastError()
    left = lib.hipSetDevice(1 << 20)  # no such device; refused by the runtime on the host
    codes_returned = [c() for c in calls]
    stays = lib.hipGetLastError()
    assert left != 0 and stays == left
    assert codes_returned == [bk.RKB_OK] * len(calls)
    torch.cuda.synchronize()
    assert torch.equal(h, bk.rkb_gated_fwd(x, wg, wu)[0]) and torch.equal(dx, bk.rkb_gated_bwd(dh, x, wg, wu)[0])


def test_layer_norm_of_more_rows_than_a_launch_has_blocks():
    """Wide rows take a block of 1024 lanes each, and 2^22 such blocks pass 32 bits of lanes; one row stands for all."""
    rows, cols = (1 << 22) + 3, 8200
    x, w = rand(1, cols, seed=1, dtype=BF), rand(cols, seed=2, dtype=BF)
    want = bk.rkb_layer_norm_fwd(x, w)
    got = bk.rkb_layer_norm_fwd(x.expand(rows, cols), w)
    for at in (0, (1 << 20) - 1, 1 << 20, (1 << 21) + 1, (1 << 22) - 1, 1 << 22, rows - 1):
        assert all(torch.equal(p[at], q[0]) for p, q in zip(got, want)), at
    assert bool((got[1] == want[1]).all()) and bool((got[2] == want[2]).all())
