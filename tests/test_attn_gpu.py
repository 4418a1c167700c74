"""Attention, its bias and the 8-bit cache (paper_2307_01236_amd/block.py) on an MI355X against their 64-bit definitions, within the
bounds that 32-bit sums and the stated roundings allow (attn_oracle)."""
import ctypes
import math

import pytest
import torch

import attn_oracle as ao
from paper_2307_01236_amd import block as bk

pytestmark = pytest.mark.gpu
BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def rand(*shape, seed=0, dtype=FP, scale=1.0):
    t = torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale
    return t.to(dtype).cuda()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def problem(B, Q, T, H, K, D, dtype, lens=None, mask=False, causal=False, firsts=None, bias=None, seed=0):
    """q, k, v, do and the keyword arguments of both the operators and the oracle.  bias: (buckets, max_distance, two_sided, type)."""
    q, k, v = rand(B, Q, H, D, seed=seed + 1, dtype=dtype), rand(B, T, K, D, seed=seed + 2, dtype=dtype), rand(B, T, K, D, seed=seed + 3, dtype=dtype)
    do = rand(B, Q, H, D, seed=seed + 4, dtype=dtype, scale=0.1)
    how, want = dict(causal=causal), dict(causal=causal)
    if lens is not None:
        how["lens"], want["lens"] = ints(lens), lens
    if mask:
        m = torch.rand(B, T, generator=torch.Generator().manual_seed(seed + 5)) < 0.7
        how["mask"], want["mask"] = m.cuda(), m
    if firsts is not None:
        how["first"], want["firsts"] = firsts if isinstance(firsts, int) else ints(firsts), firsts
    if bias is not None:
        n, far, two, t = bias
        table = rand(n, H, seed=seed + 6, dtype=t)
        how["bias"] = bk.RelBias(table, far, two)
        want.update(table=table, max_distance=far, two_sided=two)
    return (q, k, v, do), how, ao.Case(q, k, v, **want)


def check_step(tensors, how, case, keep="16bit"):
    q, k, v, do = tensors
    dtype = q.dtype
    o, kept = bk.rkb_attn_fwd(q, k, v, keep=keep, **how)
    want = case.forward()
    bounds = case.forward_bounds(dtype)
    assert ao.worst(o, want[0], bounds[0]) <= 1.0
    if keep != "none":
        assert ao.worst(kept[1], want[1], bounds[1]) <= 1.0
    if keep == "full":
        assert kept[0].dtype == FP and ao.worst(kept[0], want[0], case.forward_bounds(dtype, FP)[0]) <= 1.0
    got = bk.rkb_attn_bwd(do, q, k, v, kept, **how)
    table_dtype = how["bias"].table.dtype if "bias" in how else None
    refs = case.backward(do)[0]
    limits = case.backward_bounds(do, dtype, dtype if keep == "16bit" else FP, table_dtype)
    for name, g, r, e in zip(("dq", "dk", "dv", "dtable"), got, refs, limits):
        assert (g is None) == (r is None), name
        if r is not None:
            assert ao.worst(g, r, e) <= 1.0, name


# B, Q, T, heads, key heads, width, and what else
SHAPES = {
    "one": (1, 1, 1, 1, 1, 1, {}),
    "token": (1, 1, 128, 8, 8, 64, {}),
    "tokens": (3, 2, 333, 8, 2, 80, dict(lens=[333, 17, 0])),
    "many_heads": (1, 1, 500, 40, 1, 128, {}),  # more rows of a key head than a workgroup has
    "splits": (2, 1, 3001, 4, 2, 64, dict(lens=[3001, 700])),
    "tile": (1, 128, 64, 2, 2, 64, {}),
    "past_a_tile": (2, 129, 65, 3, 3, 40, {}),
    "short_keys": (2, 300, 3, 2, 1, 128, {}),
    "one_key": (2, 70, 1, 2, 2, 32, {}),
    "ragged": (3, 200, 171, 4, 2, 72, dict(lens=[171, 1, 64], mask=True)),
    "odd_width": (2, 97, 66, 2, 2, 13, dict(mask=True)),
    "wide": (1, 130, 100, 2, 1, 256, dict(lens=[99])),
    "wide_odd": (1, 70, 75, 2, 2, 201, {}),
    "wide_few": (1, 3, 700, 4, 2, 192, {}),
    "long_keys": (1, 65, 1500, 2, 2, 64, dict(mask=True)),
    "causal": (2, 150, 150, 2, 1, 64, dict(causal=True)),
    "causal_behind": (2, 90, 200, 2, 2, 32, dict(causal=True, firsts=[110, -30])),
    "causal_far": (1, 40, 60, 1, 1, 16, dict(causal=True, firsts=1 << 35)),
    "bias_two": (2, 140, 140, 2, 2, 64, dict(bias=(32, 128, True, FP))),
    "bias_ragged": (2, 190, 333, 4, 2, 40, dict(bias=(10, 50, True, None), lens=[333, 100], mask=True)),
    "bias_one": (1, 257, 257, 2, 1, 128, dict(bias=(32, 128, False, None), causal=True)),
    "bias_far": (1, 100, 1300, 1, 1, 16, dict(bias=(128, 1024, True, FP), firsts=600)),
    "bias_least": (1, 70, 80, 2, 2, 8, dict(bias=(2, 2, False, FP))),
    "bias_wide": (1, 66, 70, 1, 1, 256, dict(bias=(14, 300, True, FP), firsts=[5])),
    "bias_token": (3, 1, 400, 6, 2, 64, dict(bias=(32, 128, False, FP), causal=True, firsts=[399, 10, -1], lens=[400, 11, 0])),
    "bias_group": (2, 100, 64, 6, 2, 24, dict(bias=(8, 20, True, FP))),
}


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("name", SHAPES)
def test_step(name, dtype):
    *sizes, more = SHAPES[name]
    more = dict(more)
    if more.get("bias") and more["bias"][3] is None:
        more["bias"] = more["bias"][:3] + (dtype,)
    check_step(*problem(*sizes, dtype, **more))


@pytest.mark.parametrize("keep", ["none", "16bit", "full"])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_what_is_kept(keep, dtype):
    check_step(*problem(2, 131, 150, 4, 2, 64, dtype, bias=(16, 40, True, FP), lens=[150, 90]), keep=keep)


def test_what_is_kept_changes_no_output():
    (q, k, v, do), how, _ = problem(2, 131, 150, 4, 2, 64, BF, bias=(16, 40, True, FP))
    outs = [bk.rkb_attn_fwd(q, k, v, keep=keep, **how) for keep in ("none", "16bit", "full")]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][0], outs[2][0]) and torch.equal(outs[1][1][1], outs[2][1][1])
    assert outs[0][1] is None and outs[1][1][0] is outs[1][0] and torch.equal(outs[2][1][0].to(BF), outs[0][0])
    made_again, full = bk.rkb_attn_bwd(do, q, k, v, None, **how), bk.rkb_attn_bwd(do, q, k, v, outs[2][1], **how)
    assert all(torch.equal(a, b) for a, b in zip(made_again, full))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_large_and_small_values(dtype):
    """Scores that differ by hundreds, so that maxima move late and probabilities vanish; gradients near the type's ends."""
    (q, k, v, do), how, _ = problem(1, 140, 300, 2, 2, 64, dtype)
    k = k * torch.linspace(0.1, 30.0, 300, device="cuda")[None, :, None, None].to(dtype)  # maxima rise along the keys
    for scale in (1e-5, 1.0, 300.0):
        d = (do.float() * scale).to(dtype)
        check_step((q, k, v, d), how, ao.Case(q, k, v))


def test_scale_is_taken_as_given():
    (q, k, v, do), _, _ = problem(1, 70, 90, 2, 2, 64, BF)
    check_step((q, k, v, do), dict(scale=0.02), ao.Case(q, k, v, scale=0.02))


# ------------------------------------------------------------------ what must not matter

def test_rows_without_keys_are_zero():
    (q, k, v, do), _, _ = problem(3, 80, 100, 2, 2, 64, BF)
    for how in (dict(lens=ints([0, 100, 0])), dict(mask=torch.zeros(3, 100, dtype=torch.bool, device="cuda")),
                dict(causal=True, first=-40), dict(lens=ints([-5, 0, 1 << 30]))):
        o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit", **how)
        empty = (kept[1] == -math.inf).transpose(1, 2)
        assert bool(empty.any()) and bool(o.isfinite().all()) and not o[empty].any()
        grads = bk.rkb_attn_bwd(do, q, k, v, kept, **how)
        assert all(bool(g.isfinite().all()) for g in grads[:3]) and not grads[0][empty].any()
    small = bk.rkb_attn_fwd(q[:, :1], k, v, lens=ints([0, 100, 0]), keep="16bit")  # the form for few rows
    assert not small[0][0].any() and bool((small[1][1][2] == -math.inf).all()) and bool(small[0][1].any())


@pytest.mark.parametrize("Q", [1, 100])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -3.0e38])
def test_dead_places_are_not_looked_at(Q, value):
    (q, k, v, do), how, _ = problem(2, Q, 150, 4, 2, 64, BF, lens=[149, 70], mask=True, bias=(8, 30, True, FP))
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit", **how)
    want = bk.rkb_attn_bwd(do, q, k, v, kept, **how)
    dead = ~how["mask"].clone()
    dead[0, 149:] = True
    dead[1, 70:] = True
    k2, v2 = k.clone(), v.clone()
    k2[dead], v2[dead] = value, value
    o2, kept2 = bk.rkb_attn_fwd(q, k2, v2, keep="16bit", **how)
    assert torch.equal(o, o2) and torch.equal(kept[1], kept2[1])
    got = bk.rkb_attn_bwd(do, q, k2, v2, kept2, **how)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and not got[1][dead].any() and not got[2][dead].any()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("B,Q,T,H,K,D,more", [
    (2, 70, 70, 4, 2, 64, dict(mask="left", causal=True)), (2, 200, 190, 2, 2, 128, dict(causal=True, firsts=[-40, -300])),
    (1, 40, 50, 2, 1, 200, dict(causal=True, firsts=-9)), (2, 150, 40, 2, 2, 40, dict(lens=[40, 0], bias=(8, 16, True, FP))),
    (2, 300, 300, 4, 4, 64, dict(mask="left", causal=True, bias=(32, 128, True, FP)))])
def test_queries_without_keys_are_not_looked_at(B, Q, T, H, K, D, more, value, dtype):
    more = dict(more)
    left = more.pop("mask", None)
    (q, k, v, do), how, _ = problem(B, Q, T, H, K, D, dtype, **more)
    if left:
        how["mask"] = torch.arange(T, device="cuda") >= torch.tensor([[37], [5]], device="cuda")
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="full", **how)
    dead = (kept[1] == -math.inf).permute(0, 2, 1)  # [B, Q, H]
    assert dead.any() and not dead.all()
    want = bk.rkb_attn_bwd(do.masked_fill(dead[..., None], 0), q.masked_fill(dead[..., None], 0), k, v, kept, **how)
    q, do = q.masked_fill(dead[..., None], value), do.masked_fill(dead[..., None], value)
    o2, kept2 = bk.rkb_attn_fwd(q, k, v, keep="full", **how)
    assert torch.equal(o, o2) and torch.equal(kept[1], kept2[1])
    for a, b in zip(want, bk.rkb_attn_bwd(do, q, k, v, kept, **how)):
        assert (a is None and b is None) or (torch.equal(a, b) and bool(a.isfinite().all()))


def test_bad_values_stay_in_their_row_and_head():
    (q, k, v, do), _, _ = problem(2, 100, 90, 4, 4, 64, BF)
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit")
    q2 = q.clone()
    q2[0, 37, 1, 5] = float("nan")
    q2[1, 99, 3, 0] = float("inf")
    o2, kept2 = bk.rkb_attn_fwd(q2, k, v, keep="16bit")
    bad = torch.zeros(2, 100, 4, dtype=torch.bool, device="cuda")
    bad[0, 37, 1] = bad[1, 99, 3] = True
    assert bool(o2[bad].isnan().any(1).all()) and torch.equal(o2[~bad], o[~bad])
    dq, dk, dv, _ = bk.rkb_attn_bwd(do, q2, k, v, kept2)
    assert bool(dq[~bad].isfinite().all()) and bool(dk[0, :, 1].isnan().any()) and bool(dk[0, :, 0].isfinite().all())


@pytest.mark.parametrize("Q", [1, 100])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_bias_entries_at_the_ends(dtype, Q):
    """An entry of -inf, or of a type's lowest value, hides its keys as a mask does (not f16's, which 32 bits tell apart)."""
    (q, k, v, do), how, _ = problem(1, Q, 120, 2, 2, 64, dtype, bias=(8, 20, True, FP), firsts=10)
    table = how["bias"].table
    for low in (-math.inf, torch.finfo(FP).min, torch.finfo(BF).min, -1e30, -65504.0):
        table[3], table[7, 1] = low, low
        check_step((q, k, v, do), how, ao.Case(q, k, v, table=table, max_distance=20, two_sided=True, firsts=10))
    for low in (-math.inf, torch.finfo(FP).min):
        table[:] = low
        o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit", **how)
        assert not o.any() and bool((kept[1] == -math.inf).all())
        assert not any(bool(g.any()) for g in bk.rkb_attn_bwd(do, q, k, v, kept, **how))


def spread(t, seed):
    """The same values as a view with other strides: heads before rows, an odd start, gaps."""
    B, R, H, D = t.shape
    wide = torch.full((H + 1, B, R + 2, D + 3), float("nan"), dtype=t.dtype, device=t.device).flatten()
    wide = torch.cat([wide[:1], wide])[1 if seed % 2 else 0:][:(H + 1) * B * (R + 2) * (D + 3)].view(H + 1, B, R + 2, D + 3)
    view = wide[:H, :, 1:R + 1, 1:D + 1].permute(1, 2, 0, 3)
    view.copy_(t)
    return view


@pytest.mark.parametrize("Q,T,D", [(1, 300, 64), (5, 40, 33), (130, 90, 64), (70, 200, 40), (66, 70, 201)])
def test_strides_do_not_matter(Q, T, D):
    (q, k, v, do), how, _ = problem(2, Q, T, 4, 2, D, HF, mask=True)
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="full", **how)
    want = bk.rkb_attn_bwd(do, q, k, v, kept, **how)
    q2, k2, v2, d2 = (spread(t, s) for s, t in enumerate((q, k, v, do)))
    mask = torch.ones(2, T + 5, dtype=torch.bool, device="cuda")
    mask[:, 3:T + 3] = how["mask"]
    how2 = dict(mask=mask[:, 3:T + 3])
    o2, kept2 = bk.rkb_attn_fwd(q2, k2, v2, keep="full", **how2)
    assert torch.equal(o, o2) and torch.equal(kept[0], kept2[0]) and torch.equal(kept[1], kept2[1])
    assert all(torch.equal(a, b) for a, b in zip(bk.rkb_attn_bwd(d2, q2, k2, v2, kept2, **how2)[:3], want[:3]))


def test_heads_of_one_tensor_and_broadcast_keys():
    """q, k and v as views of one projection's output; keys that all sequences share (stride 0)."""
    x = rand(2, 90, 3, 4, 64, dtype=BF)
    q, k, v = x[:, :, 0], x[:, :, 1], x[:, :, 2]
    want = bk.rkb_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous())[0]
    assert torch.equal(bk.rkb_attn_fwd(q, k, v)[0], want)
    k1, v1 = k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1)
    do = rand(2, 90, 4, 64, seed=9, dtype=BF)
    a = bk.rkb_attn_bwd(do, q, k1, v1)
    b = bk.rkb_attn_bwd(do, q, k1.contiguous(), v1.contiguous())
    assert all(torch.equal(s, t) for s, t in zip(a[:3], b[:3]))


def test_results_are_the_same_every_time_and_in_any_batch():
    (q, k, v, do), how, _ = problem(3, 150, 260, 4, 2, 64, HF, bias=(32, 128, True, FP))
    first = (bk.rkb_attn_fwd(q, k, v, **how)[0], *bk.rkb_attn_bwd(do, q, k, v, **how))
    for _ in range(3):
        again = (bk.rkb_attn_fwd(q, k, v, **how)[0], *bk.rkb_attn_bwd(do, q, k, v, **how))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_outputs_into_a_wider_tensor():
    """At the C interface: outputs with strides of their own, and nothing written beside them."""
    lib, st = bk.load(), torch.cuda.current_stream().cuda_stream
    (q, k, v, do), _, _ = problem(2, 70, 45, 3, 3, 20, BF)
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit")
    want = bk.rkb_attn_bwd(do, q, k, v, kept)
    a = bk.CAttn(bk.RKB_BF16, 0, 2, 70, 45, 3, 3, 20, 20 ** -0.5, 0, None, None, None, 0, None, 0, 0, 0, 0)

    def place(rows):
        t = torch.full((2, rows + 3, 4, 29), 7.0, dtype=BF, device="cuda")
        return t, t[:, 1:rows + 1, :3, 5:25], bk.CHeads(t[:, 1:, :, 5:].data_ptr(), *t.stride()[:3])

    def at(t):
        return bk.CHeads(t.data_ptr(), *t.stride()[:3])

    n = ctypes.c_size_t(0)
    assert lib.rkb_attn_fwd_workspace(a, 0, 0, n) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    whole, view, out = place(70)
    assert lib.rkb_attn_fwd(a, at(q), at(k), at(v), None, out, None, None, ws.data_ptr(), n.value, st) == 0
    assert torch.equal(view, o)
    view.fill_(7.0)
    assert bool((whole == 7.0).all())
    assert lib.rkb_attn_bwd_workspace(a, 0, 0, n) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    outs = [place(70), place(45), place(45)]
    assert lib.rkb_attn_bwd(a, at(do), at(q), at(k), at(v), at(o), None, kept[1].data_ptr(), *(x[2] for x in outs), None, ws.data_ptr(), n.value, st) == 0
    for (whole, view, _), w in zip(outs, want):
        assert torch.equal(view, w)
        view.fill_(7.0)
        assert bool((whole == 7.0).all())
    # dk and dv alone, and dq alone, are the same
    none = bk.CHeads(None, 0, 0, 0)
    outs = [place(70), place(45), place(45)]
    for which in ((outs[0][2], none, none), (none, outs[1][2], outs[2][2])):
        assert lib.rkb_attn_bwd(a, at(do), at(q), at(k), at(v), at(o), None, kept[1].data_ptr(), *which, None, ws.data_ptr(), n.value, st) == 0
    assert all(torch.equal(x[1], w) for x, w in zip(outs, want))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_gradients_one_at_a_time(dtype):
    """At the C interface, of a call whose keys are split: each alone is what it is with the others."""
    lib, st = bk.load(), torch.cuda.current_stream().cuda_stream
    (q, k, v, do), how, _ = problem(1, 70, 1100, 4, 2, 72, dtype, lens=[1030], bias=(8, 20, True, FP))
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit", **how)
    want = bk.rkb_attn_bwd(do, q, k, v, kept, **how)
    table = how["bias"].table
    a = bk.CAttn(bk.RKB_BF16 if dtype == BF else bk.RKB_F16, 0, 1, 70, 1100, 4, 2, 72, 72 ** -0.5, 0, None, how["lens"].data_ptr(), None, 0,
                 table.data_ptr(), bk.RKB_F32, 8, 20, 1)

    def at(t):
        return bk.CHeads(t.data_ptr(), *t.stride()[:3])

    n, none = ctypes.c_size_t(0), bk.CHeads(None, 0, 0, 0)
    assert lib.rkb_attn_bwd_workspace(a, 0, 1, n) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    for asked in ((0,), (1, 2), (3,), (0, 3), (0, 1, 2)):
        got = [torch.empty_like(w) for w in want]
        outs = [at(got[i]) if i in asked else none for i in range(3)]
        assert lib.rkb_attn_bwd(a, at(do), at(q), at(k), at(v), at(o), None, kept[1].data_ptr(), *outs, got[3].data_ptr() if 3 in asked else None,
                                ws.data_ptr(), n.value, st) == 0
        assert all(torch.equal(got[i], want[i]) for i in asked), asked


def test_empty_tensors():
    q, k = rand(0, 5, 2, 16, dtype=BF), rand(0, 7, 2, 16, dtype=BF)
    assert bk.rkb_attn_fwd(q, k, k)[0].shape == q.shape
    table = rand(8, 2)
    dq, dk, dv, dt = bk.rkb_attn_bwd(q, q, k, k, bias=bk.RelBias(table, 20))
    assert dq.shape == q.shape and dk.shape == k.shape and not dt.any()
    q, k = rand(2, 5, 2, 16, dtype=BF), rand(2, 0, 2, 16, dtype=BF)
    o, kept = bk.rkb_attn_fwd(q, k, k, keep="16bit")
    assert not o.any() and bool((kept[1] == -math.inf).all())
    dq, dk, _, dt = bk.rkb_attn_bwd(q, q, k, k, kept, bias=bk.RelBias(table, 20))
    assert not dq.any() and dk.shape == k.shape and not dt.any()
    q, k = rand(2, 0, 2, 16, dtype=HF), rand(2, 7, 2, 16, dtype=HF)
    o, kept = bk.rkb_attn_fwd(q, k, k, keep="16bit")
    dq, dk, dv, _ = bk.rkb_attn_bwd(q, q, k, k, kept)
    assert o.shape == q.shape and not dk.any() and not dv.any()


def test_the_binding_refuses_what_does_not_fit():
    q, k = rand(2, 5, 4, 16, dtype=BF), rand(2, 7, 2, 16, dtype=BF)
    cache = bk.Kv8.zeros(2, 40, 2, 16)
    table = rand(8, 4)
    kept = bk.rkb_attn_fwd(q, k, k, keep="16bit")[1]
    for call in (lambda: bk.rkb_attn_fwd(q.half(), k, k), lambda: bk.rkb_attn_fwd(q, k, k[:, :6]), lambda: bk.rkb_attn_fwd(q, k[:1], k[:1]),
                 lambda: bk.rkb_attn_fwd(q, k, k[..., :8]), lambda: bk.rkb_attn_fwd(q[..., ::2], k, k), lambda: bk.rkb_attn_fwd(q, k),
                 lambda: bk.rkb_attn_fwd(q[0], k, k), lambda: bk.rkb_attn_fwd(q.float(), k.float(), k.float()),
                 lambda: bk.rkb_attn_fwd(q[:, :, :3], k, k), lambda: bk.rkb_attn_fwd(q, k, k, scale=-1.0),
                 lambda: bk.rkb_attn_fwd(q, k, k, lens=torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: bk.rkb_attn_fwd(q, k, k, lens=ints([1])),
                 lambda: bk.rkb_attn_fwd(q, k, k, mask=torch.ones(2, 6, dtype=torch.bool, device="cuda")),
                 lambda: bk.rkb_attn_fwd(q, k, k, mask=torch.ones(2, 7, device="cuda")), lambda: bk.rkb_attn_fwd(q, k, k, first=ints([1, 2, 3])),
                 lambda: bk.rkb_attn_fwd(q, k, k, bias=table), lambda: bk.rkb_attn_fwd(q, k, k, bias=bk.RelBias(table[:, :3], 20)),
                 lambda: bk.rkb_attn_fwd(q, k, k, bias=bk.RelBias(table[:7], 20)), lambda: bk.rkb_attn_fwd(q, k, k, bias=bk.RelBias(table, 2000)),
                 lambda: bk.rkb_attn_fwd(q, cache, k), lambda: bk.rkb_attn_fwd(q.half(), cache), lambda: bk.rkb_attn_fwd(q[:1], cache),
                 lambda: bk.rkb_attn_bwd(q, q, k, k, (kept[0],)), lambda: bk.rkb_attn_bwd(q, q, k, k, (kept[0], kept[1][:, :3])),
                 lambda: bk.rkb_attn_bwd(q[:, :4], q, k, k), lambda: bk.rkb_attn_bwd(q, q, cache, k), lambda: bk.rkb_kv8_write(cache, k, k[:, :3]),
                 lambda: bk.rkb_kv8_write(cache, k.half(), k.half()), lambda: bk.rkb_kv8_write(cache, q, q), lambda: bk.rkb_kv8_write(cache, k, k, ints([1])),
                 lambda: bk.rkb_kv8_load(bk.Kv8(cache.codes, cache.exps, (2, 70, 2, 16), BF))):
        with pytest.raises(bk.RKBError) as e:
            call()
        assert e.value.code == bk.RKB_E_INVAL


# ------------------------------------------------------------------ the cache

def caches(B, tokens, K, D, dtype):
    return bk.Kv8.zeros(B, tokens, K, D, dtype), [[[ao.Cache(tokens, D, dtype) for _ in range(K)] for _ in range(B)] for _ in range(2)]


def check_cache(cache, want):
    """Codes, exponents and values are those of the definition."""
    codes, exps = cache.codes.cpu(), cache.exps.cpu()
    values = [x.cpu().double() for x in bk.rkb_kv8_load(cache)]
    _, B, K = codes.shape[:3]
    for side in range(2):
        for b in range(B):
            for h in range(K):
                w = want[side][b][h]
                assert exps[side, b, h].tolist() == w.exps, (side, b, h)
                assert not codes[side, b, h, :, w.dim:].any()
                fine = torch.tensor([e != 255 for e in w.exps]).repeat_interleave(32)
                assert torch.equal(codes[side, b, h, :, :w.dim].double()[fine], w.codes[fine]), (side, b, h)
                ref = w.values()
                assert torch.equal(values[side][b, :, h].nan_to_num(nan=-1.0), ref.nan_to_num(nan=-1.0))


def write(cache, want, k, v, firsts, counts=None):
    bk.rkb_kv8_write(cache, k, v, firsts if isinstance(firsts, int) else ints(firsts), None if counts is None else ints(counts))
    B, n, K, _ = k.shape
    for side, x in enumerate((k, v)):
        x = ao.d(x)
        for b in range(B):
            first = firsts if isinstance(firsts, int) else firsts[b]
            count = n if counts is None else min(max(counts[b], 0), n)
            for h in range(K):
                want[side][b][h].write(x[b, :count, h], first)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,tokens,K,D", [(1, 1, 1, 1), (2, 100, 2, 40), (3, 64, 1, 128), (1, 33, 3, 256), (2, 200, 2, 13)])
def test_cache_writes(B, tokens, K, D, dtype):
    cache, want = caches(B, tokens, K, D, dtype)
    step = 0
    for n, firsts, counts in ((tokens // 2 + 1, 0, None), (1, [tokens // 2 + 1 - b for b in range(B)], None), (40, [7 * b for b in range(B)], [40 - 13 * b for b in range(B)]),
                              (5, [tokens - 2] * B, None), (70, -3, [0 if b == 1 else 70 for b in range(B)]), (3, tokens, None)):
        k, v = (rand(B, n, K, D, seed=10 * step + s, dtype=dtype, scale=2.0 ** (3 * step - 6)) for s in (1, 2))
        write(cache, want, k, v, firsts, counts)
        check_cache(cache, want)
        step += 1


def test_cache_token_by_token():
    cache, want = caches(2, 70, 2, 24, HF)
    scales = torch.logspace(-3, 3, 70)
    for t in range(70):
        k, v = (rand(2, 1, 2, 24, seed=2 * t + s, dtype=HF, scale=float(scales[(t * 29) % 70])) for s in (0, 1))
        write(cache, want, k, v, [t, max(0, t - 5)])
    check_cache(cache, want)


def test_cache_at_the_ends_of_the_types():
    for dtype in (BF, HF):
        cache, want = caches(1, 64, 1, 32, dtype)
        top = torch.finfo(dtype).max
        x = rand(1, 40, 1, 32, seed=3, dtype=dtype)
        x[0, 3, 0, 5], x[0, 35, 0, 1] = top, float("nan")
        write(cache, want, x, x.clamp(-1e-30 if dtype == BF else -1e-7, 1e-30 if dtype == BF else 1e-7), 0)
        check_cache(cache, want)
        write(cache, want, x[:, :2], -x[:, 3:5], 32)  # a block that was NaN begins again
        check_cache(cache, want)
        write(cache, want, x[:, 35:36], x[:, :1], 40)  # and takes a NaN behind tokens that it keeps
        write(cache, want, x[:, :1], x[:, :1], 41)
        check_cache(cache, want)


def test_other_blocks_stay_as_they_were():
    cache, want = caches(2, 160, 2, 16, BF)
    cache.codes.random_(-127, 128, generator=torch.Generator("cuda").manual_seed(1))
    cache.exps.random_(100, 140, generator=torch.Generator("cuda").manual_seed(2))
    before = cache.codes.clone(), cache.exps.clone()
    k = rand(2, 20, 2, 16, dtype=BF)
    bk.rkb_kv8_write(cache, k, k, ints([40, 64]), ints([20, 0]))
    touched = torch.zeros_like(before[1], dtype=torch.bool)
    touched[:, 0, :, 1] = True
    assert torch.equal(before[1][~touched], cache.exps[~touched])
    rows = touched.repeat_interleave(32, 3)
    assert torch.equal(before[0][~rows], cache.codes[~rows])


def test_cache_rows_of_any_stride():
    k, v = rand(2, 50, 3, 40, dtype=HF), rand(2, 50, 3, 40, seed=1, dtype=HF)
    a, b = bk.Kv8.zeros(2, 64, 3, 40, HF), bk.Kv8.zeros(2, 64, 3, 40, HF)
    bk.rkb_kv8_write(a, k, v, 3)
    bk.rkb_kv8_write(b, spread(k, 0), spread(v, 1), 3)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.exps, b.exps)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,Q,T,H,K,D,more", [
    (1, 1, 1, 1, 1, 1, {}), (2, 1, 500, 16, 4, 128, dict(causal=True, firsts=[499, 100], lens=[500, 101])), (1, 3, 1000, 8, 8, 64, dict(mask=True)),
    (2, 100, 150, 4, 2, 72, dict(causal=True, firsts=[50, 20], lens=[150, 120], bias=(32, 128, False, FP))), (1, 70, 90, 2, 1, 256, {}),
    (1, 2, 300, 2, 1, 200, dict(bias=(8, 50, True, FP))), (2, 200, 129, 3, 3, 64, dict(lens=[129, 0], mask=True)), (1, 1, 33, 40, 1, 16, dict(lens=[32]))])
def test_attention_over_a_cache(B, Q, T, H, K, D, more, dtype):
    """The same bits as over the values that the cache stands for."""
    (q, k, v, _), how, _ = problem(B, Q, T, H, K, D, dtype, **more)
    cache = bk.Kv8.zeros(B, T, K, D, dtype)
    bk.rkb_kv8_write(cache, k, v)
    k8, v8 = bk.rkb_kv8_load(cache)
    want, kept = bk.rkb_attn_fwd(q, k8, v8, keep="full", **how)
    got, kept8 = bk.rkb_attn_fwd(q, cache, keep="full", **how)
    assert torch.equal(got, want) and torch.equal(kept[0], kept8[0]) and torch.equal(kept[1], kept8[1])


def test_what_lies_behind_a_length_in_a_cache_is_not_looked_at():
    (q, k, v, _), _, _ = problem(2, 1, 200, 4, 2, 64, BF)
    cache = bk.Kv8.zeros(2, 200, 2, 64)
    bk.rkb_kv8_write(cache, k, v)
    for Q in (1, 100):
        q = rand(2, Q, 4, 64, dtype=BF)
        lens = ints([64, 90])
        want = bk.rkb_attn_fwd(q, cache, lens=lens)[0]
        worse = bk.Kv8(cache.codes.clone(), cache.exps.clone(), cache.shape, cache.dtype)
        worse.exps[:, 0, :, 2:] = 255
        worse.exps[:, 1, :, 3:] = 255
        worse.codes[:, 1, :, 90:] = 127
        assert torch.equal(bk.rkb_attn_fwd(q, worse, lens=lens)[0], want)
        worse.exps[1, 1, 0, 0] = 255  # a block that stands for NaN, among the live ones, of one key head's values
        out = bk.rkb_attn_fwd(q, worse, lens=lens)[0]
        assert bool(out[1, :, :2].isnan().all()) and torch.equal(out[1, :, 2:], want[1, :, 2:]) and torch.equal(out[0], want[0])


# ------------------------------------------------------------------ as they are used

def test_a_prompt_and_then_token_by_token():
    """A prompt in pieces, then single tokens: each query over a cache that grows, with a bias, against the definition on what the cache
    holds then.  One sequence is longer than the other."""
    B, H, K, D, total, bias_args = 2, 4, 2, 64, 120, (16, 60, False, FP)
    (q, k, v, _), how, _ = problem(B, total, total, H, K, D, BF, bias=bias_args)
    cache = bk.Kv8.zeros(B, total, K, D)
    at = [0, 0]
    for n, counts in ((70, [70, 41]), (30, [30, 0]), *(((1, [1, 1]),) * 9)):
        pick = lambda x: torch.stack([torch.cat([x[b, at[b]:at[b] + n], x.new_zeros(max(0, n - len(x[b, at[b]:])), *x.shape[2:])]) for b in range(B)])  # noqa: E731
        bk.rkb_kv8_write(cache, pick(k), pick(v), ints(at), ints(counts))
        lens = [a + c for a, c in zip(at, counts)]
        o = bk.rkb_attn_fwd(pick(q), cache, lens=ints(lens), causal=True, first=ints(at), bias=how["bias"])[0]
        k8, v8 = bk.rkb_kv8_load(cache)
        case = ao.Case(pick(q), k8, v8, lens=lens, causal=True, firsts=at, table=how["bias"].table, max_distance=60, two_sided=False)
        ref, bound = case.forward()[0], case.forward_bounds(BF)[0]
        for b in range(B):
            assert ao.worst(o[b, :counts[b]], ref[b, :counts[b]], bound[b, :counts[b]]) <= 1.0
        at = lens


def test_a_block_with_kept_values_in_8_bits():
    """Layer norm, projections, attention, and back: the gradients by the operators against 64-bit autograd, with q, k and v as the operators
    had them; then with keys and values kept in a cache between the passes."""
    B, T, S, H, D, W = 2, 90, 70, 4, 32, 128
    x, ctx = rand(B, T, W, seed=1, dtype=BF), rand(B, S, W, seed=2, dtype=BF)
    w = [rand(W, W, seed=3 + i, dtype=BF, scale=W ** -0.5) for i in range(3)]
    n, mean, rstd = bk.rkb_layer_norm_fwd(x)
    q, k, v = (y.view(B, -1, H, D) for y in (n @ w[0].t(), ctx @ w[1].t(), ctx @ w[2].t()))
    o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit")
    do = rand(B, T, H, D, seed=9, dtype=BF)
    dq, dk, dv, _ = bk.rkb_attn_bwd(do, q, k, v, kept)
    dwq = bk.rkb_weight_grad(dq.flatten(2), n)
    dx = bk.rkb_layer_norm_bwd(dq.flatten(2) @ w[0], x, mean, rstd)[0]
    xd, wd = ao.d(x).requires_grad_(), [ao.d(t).requires_grad_() for t in w]
    cd = ao.d(ctx)
    nd = torch.nn.functional.layer_norm(xd, (W,), eps=1e-5)
    qd, kd, vd = (y.view(B, -1, H, D).transpose(1, 2) for y in (nd @ wd[0].t(), cd @ wd[1].t(), cd @ wd[2].t()))
    p = torch.softmax(qd @ kd.transpose(2, 3) * D ** -0.5, 3)
    (p @ vd).transpose(1, 2).backward(ao.d(do))
    for got, ref in ((dwq, wd[0].grad), (dx, xd.grad), (bk.rkb_weight_grad(dk.flatten(2), ctx), wd[1].grad), (bk.rkb_weight_grad(dv.flatten(2), ctx), wd[2].grad)):
        # each of the half a dozen roundings on the way is at most 2^-8, and they add up as independent ones at worst linearly
        assert float((ao.d(got) - ref).norm() / ref.norm()) <= 6 * 2.0 ** -8
    cache = bk.Kv8.zeros(B, S, H, D)
    bk.rkb_kv8_write(cache, k, v)
    assert cache.nbytes() == 2 * B * H * (96 * D + 3)  # a byte an element of 96 tokens, and one for each 32 tokens
    k8, v8 = bk.rkb_kv8_load(cache)
    o8, kept8 = bk.rkb_attn_fwd(q, cache, keep="16bit")
    check_step((q, k8, v8, do), {}, ao.Case(q, k8, v8))
    again = bk.rkb_attn_bwd(do, q, k8, v8, kept8)
    assert all(bool(g.isfinite().all()) for g in again[:3])


def test_graphs_of_steps_and_tokens():
    """Captured and replayed several times with new values in place, eager work between; two graphs at once."""
    (q, k, v, do), how, _ = problem(2, 130, 700, 4, 2, 64, HF, bias=(32, 128, True, FP), lens=[700, 300])
    cache = bk.Kv8.zeros(2, 800, 2, 64, HF)
    bk.rkb_kv8_write(cache, k, v)
    tok = rand(2, 1, 2, 64, seed=20, dtype=HF)
    at = ints([700, 300])

    def train():
        o, kept = bk.rkb_attn_fwd(q, k, v, keep="16bit", **how)
        return (o, kept[1], *bk.rkb_attn_bwd(do, q, k, v, kept, **how))

    def token():
        bk.rkb_kv8_write(cache, tok, tok, at)
        return (bk.rkb_attn_fwd(q[:, :1], cache, lens=at + 1)[0], cache.codes.clone(), cache.exps.clone())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train(), token()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for f in (train, token):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = f()
        graphs.append((g, outs, f))
    for step in range(4):
        for t, s in ((q, 1), (k, 2), (do, 3), (tok, 4)):
            t.copy_(rand(*t.shape, seed=100 * step + s, dtype=HF))
        how["bias"].table.copy_(rand(32, 4, seed=step))
        at.add_(3)
        state = cache.codes.clone(), cache.exps.clone()
        for g, outs, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in outs] for _, outs, _ in graphs]
        cache.codes.copy_(state[0])
        cache.exps.copy_(state[1])
        for (_, _, f), replayed in zip(graphs, got):
            assert all(torch.equal(a, b) for a, b in zip(f(), replayed)), step


def test_streams():
    """Queued on the current stream, behind what it waits for."""
    (q, k, v, do), how, _ = problem(2, 200, 300, 4, 2, 64, BF, bias=(32, 128, True, FP))
    want = (bk.rkb_attn_fwd(q, k, v, **how)[0], *bk.rkb_attn_bwd(do, q, k, v, **how))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            late = torch.zeros_like(q)
            torch.cuda._sleep(2_000_000)
            late.copy_(q)
            outs.append((bk.rkb_attn_fwd(late, k, v, **how)[0], *bk.rkb_attn_bwd(do, late, k, v, **how)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in outs for a, b in zip(out, want))


def test_offsets_past_32_bits():
    """A cache, and keys, of more than 2^32 elements: the last sequence is the same as alone."""
    B, T, K, D = 5, 4_200_000, 2, 128
    cache = bk.Kv8.zeros(B, T, K, D)
    k = rand(B, 40, K, D, dtype=BF)
    bk.rkb_kv8_write(cache, k, k, T - 50)
    lens, firsts = ints([T] * B), T - 11
    q = rand(B, 1, 4, D, seed=1, dtype=BF)
    mask = torch.zeros(B, T, dtype=torch.bool, device="cuda")
    mask[:, T - 50:T - 10] = True
    o = bk.rkb_attn_fwd(q, cache, lens=lens, mask=mask, causal=True, first=firsts)[0]
    small = bk.Kv8.zeros(B, 64, K, D)
    start = (T - 50) % 32
    bk.rkb_kv8_write(small, k, k, start)
    k8, v8 = bk.rkb_kv8_load(small)
    case = ao.Case(q, k8[:, start:start + 40], v8[:, start:start + 40])
    ref, bound = case.forward()[0], case.forward_bounds(BF)[0]
    assert ao.worst(o, ref, bound) <= 1.0
    del cache, mask
    wide = torch.zeros(3, 1_000_000, 12, 64, dtype=BF, device="cuda")  # 2.3e9 elements
    wide[2, -300:] = rand(300, 12, 64, seed=4, dtype=BF)
    kk, vv = wide[:, :, 0:2], wide[:, :, 2:4]
    qq = rand(3, 1, 2, 64, seed=5, dtype=BF)
    mask = torch.zeros(3, 1_000_000, dtype=torch.bool, device="cuda")
    mask[:, -300:] = True
    o = bk.rkb_attn_fwd(qq, kk, vv, mask=mask)[0]
    case = ao.Case(qq[2:], kk[2:, -300:], vv[2:, -300:])
    assert ao.worst(o[2:], case.forward()[0], case.forward_bounds(BF)[0]) <= 1.0
