"""The 64-bit definitions of the block operators: gradients against differences, checkpoints
against their properties, and planted mistakes that the comparison must notice."""
import math

import pytest
import torch

import block_oracle as bo


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def difference(f, x, v, h=1e-5):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 40)])
def test_layer_norm_gradient_is_the_difference(rows, cols):
    x, w, b, dy = rand(rows, cols), rand(cols, seed=1), rand(cols, seed=2), rand(rows, cols, seed=3)
    _, mean, rstd = bo.layer_norm(x, w, b, 1e-5)
    dx, dw, db = bo.layer_norm_grads(dy, x, mean, rstd, w)
    for grad, at, f in ((dx, x, lambda t: (bo.layer_norm(t, w, b, 1e-5)[0] * dy).sum()),
                        (dw, w, lambda t: (bo.layer_norm(x, t, b, 1e-5)[0] * dy).sum()),
                        (db, b, lambda t: (bo.layer_norm(x, w, t, 1e-5)[0] * dy).sum())):
        v = rand(*at.shape, seed=9)
        want = float((grad * v).sum())
        scale = float((grad.abs() * v.abs()).sum()) + 1.0
        assert abs(float(difference(f, at, v)) - want) < 1e-6 * scale


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_gradient_is_the_difference(kind):
    x, wg, wu, dh = rand(4, 6), rand(9, 6, seed=1), rand(9, 6, seed=2), rand(4, 9, seed=3)
    _, g, u = bo.gated(x, wg, wu, kind)
    dx, dwg, dwu, h = bo.gated_grads(dh, x, wg, wu, kind, g, u)
    assert torch.equal(h, bo.gated(x, wg, wu, kind)[0])
    for grad, at, f in ((dx, x, lambda t: (bo.gated(t, wg, wu, kind)[0] * dh).sum()),
                        (dwg, wg, lambda t: (bo.gated(x, t, wu, kind)[0] * dh).sum()),
                        (dwu, wu, lambda t: (bo.gated(x, wg, t, kind)[0] * dh).sum())):
        v = rand(*at.shape, seed=9)
        want = float((grad * v).sum())
        assert abs(float(difference(f, at, v)) - want) < 1e-7 * float((grad.abs() * v.abs()).sum() + 1)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_act_slope_stays_within_the_bounds_constants(kind):
    g = torch.linspace(-30, 30, 60001, dtype=torch.float64)
    a, s = bo.act(g, kind)
    assert float(s.abs().max()) < 1.2 and float(difference(lambda t: bo.act(t, kind)[1], g, 1.0).abs().max()) < 1.0


def test_checkpoint_properties():
    x = rand(6, 100) * torch.exp(3 * rand(6, 1, seed=4))
    x[2] = 0
    x[3, :40] = 127 * 2.0 ** -3  # the largest code exactly
    q, e, v = bo.ckpt(x, torch.float32)
    step = torch.exp2(e).repeat_interleave(32, 1)[:, :100]
    assert float(q.abs().max()) == 127 and bool((v == q * step).all())
    assert bool(((x - v).abs() <= step / 2).all())
    top = torch.stack([x[:, i:i + 32].abs().amax(1) for i in range(0, 100, 32)], 1)
    assert bool((top <= 127 * torch.exp2(e)).all())
    assert bool(((top > 127 * torch.exp2(e - 1)) | (e == -126)).all())
    assert bool((v[3, :32] == x[3, :32]).all())  # the group that is all 127 steps
    again = bo.ckpt(v, torch.float32)[2]  # the values are a fixed point
    assert torch.equal(again, v)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_checkpoint_of_the_largest_value_stays_finite(dtype):
    top = torch.finfo(dtype).max
    x = torch.full((1, 33), top, dtype=torch.float64)
    _, _, v = bo.ckpt(x, dtype)
    assert bool((v <= top).all()) and bool((v >= top * 0.98).all())
    assert torch.equal(v.to(dtype).double(), v)  # exact in the type


MISTAKES = {
    "slope without its second term": lambda g: bo.act(g, "silu")[0] / g,
    "slope of the other activation": lambda g: bo.act(g, "gelu")[1],
}


@pytest.mark.parametrize("name", MISTAKES)
def test_a_wrong_slope_is_noticed(name):
    x, wg, wu, dh = rand(8, 16), rand(32, 16, seed=1) / 4, rand(32, 16, seed=2) / 4, rand(8, 32, seed=3)
    _, g, u = bo.gated(x, wg, wu, "silu")
    dx = bo.gated_grads(dh, x, wg, wu, "silu", g, u)[0]
    bound = bo.gated_grad_bounds(dh, x, wg, wu, "silu", g, u, torch.bfloat16)[0]
    wrong = (dh * u * MISTAKES[name](g)) @ wg + (dh * bo.act(g, "silu")[0]) @ wu
    assert bo.worst(dx, dx, bound) == 0.0
    assert bo.worst(wrong, dx, bound) > 1.0


def test_a_dropped_row_and_a_wrong_mean_are_noticed():
    dy, x, w = rand(64, 48), rand(64, 48, seed=1), rand(48, seed=2)
    _, mean, rstd = bo.layer_norm(x, w, None, 1e-5)
    dx, dw, db = bo.layer_norm_grads(dy, x, mean, rstd, w)
    b = bo.layer_norm_grad_bounds(dy, x, mean, rstd, w, torch.bfloat16, torch.float32)
    fewer = bo.layer_norm_grads(dy[:-1], x[:-1], mean[:-1], rstd[:-1], w)
    assert bo.worst(fewer[1], dw, b[1]) > 1 and bo.worst(fewer[2], db, b[2]) > 1
    uncentred = rstd[:, None] * (dy * w - (x - mean[:, None]) * rstd[:, None] * (dy * w * x).mean(1, keepdim=True))
    assert bo.worst(uncentred, dx, b[0]) > 1


def test_a_step_twice_too_large_is_noticed():
    x = rand(4, 64)
    q, e, v = bo.ckpt(x, torch.float32)
    coarse = torch.round(x / torch.exp2(e + 1).repeat_interleave(32, 1)) * torch.exp2(e + 1).repeat_interleave(32, 1)
    assert not torch.equal(coarse, v)
    assert math.isfinite(float(v.abs().max()))
