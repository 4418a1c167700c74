"""The example that trains a chain of gated blocks under a plan: its gradients against a 64-bit
autograd of the same chain, and against each other over budgets."""
import os
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

import train_in_budget as ex  # noqa: E402
from paper_2307_01236_amd import rk  # noqa: E402

pytestmark = pytest.mark.gpu
LAYERS, TOKENS, WIDTH, HIDDEN = 4, 200, 136, 264


@pytest.fixture(scope="module")
def problem():
    weights = ex.make_weights(LAYERS, WIDTH, HIDDEN)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x0 = torch.randn(TOKENS, WIDTH, generator=gen, device="cuda").bfloat16()
    target = torch.randn(TOKENS, WIDTH, generator=gen, device="cuda").bfloat16()
    params = [{k: v.detach().cpu().double().requires_grad_() for k, v in w.items()} for w in weights]
    x = x0.cpu().double().requires_grad_()
    y = x
    for p in params:
        n = torch.nn.functional.layer_norm(y, (WIDTH,), p["ln_w"], p["ln_b"], 1e-5)
        y = y + (torch.nn.functional.silu(n @ p["wg"].t()) * (n @ p["wu"].t())) @ p["wd"].t()
    (0.5 * ((y - target.cpu().double()) ** 2).sum()).backward()
    return weights, x0, target, params, x.grad


def step(problem, ops, options=ex.OPTIONS):
    weights, x0, target, _, _ = problem
    grads = [{k: torch.full_like(v, float("nan")) for k, v in w.items()} for w in weights]
    dx = ex.run(ops, weights, x0, lambda y: y - target, grads, options)
    return dx, grads


def plan(problem, options, budget=None):
    weights, x0 = problem[:2]
    chain = ex.make_chain(weights[0], x0, LAYERS, slot=4096, options=options)
    s = rk.Solver(chain)
    try:
        s.solve()
        curve = s.tradeoff_curve()
        feasible = np.flatnonzero(curve != rk.RK_INF)
        s.solve(int(feasible[0]) if budget == "least" else chain.M)
        return s.schedule()[0]
    finally:
        s.close()


# Relative errors add up at most over the roundings between a weight and the loss: about ten 16-bit ones a block of 2^-9 each
# (rms), and with 8 bits three checkpoints a block whose steps are at most 1/63 of a group's largest value (about 2.6
# deviations): 2.6 / 63 / sqrt(12) each.
LIMIT_16 = 10 * LAYERS * 2.0 ** -9
LIMIT_8 = LIMIT_16 + 3 * LAYERS * 2.6 / 63 / 12 ** 0.5


@pytest.mark.parametrize("option,limit", [("16bit", LIMIT_16), ("8bit", LIMIT_8), ("none", LIMIT_16)])
def test_gradients_match_autograd(problem, option, limit):
    ops = plan(problem, (option,))
    dx, grads = step(problem, ops, (option,))
    params, dx_ref = problem[3:]
    pairs = [(dx, dx_ref)] + [(grads[b][k], params[b][k].grad) for b in range(LAYERS) for k in ex.NAMES]
    for got, ref in pairs:
        assert float((got.cpu().double() - ref).norm() / ref.norm()) <= limit


@pytest.mark.parametrize("option", ex.OPTIONS)
def test_a_tight_plan_gives_the_same_bits(problem, option):
    """Activations that are made again are the same bits, so are the gradients."""
    loose, tight = plan(problem, (option,)), plan(problem, (option,), "least")
    assert int((tight[:, 0] == rk.RK_FWD_NOSAVE).sum()) > int((loose[:, 0] == rk.RK_FWD_NOSAVE).sum())
    a, b = step(problem, loose, (option,)), step(problem, tight, (option,))
    assert torch.equal(a[0], b[0])
    assert all(torch.equal(a[1][i][k], b[1][i][k]) for i in range(LAYERS) for k in ex.NAMES)


def test_options_differ_in_what_they_keep(problem):
    weights, x0 = problem[:2]
    chain = ex.make_chain(weights[0], x0, LAYERS, slot=512)
    full, small, none = chain.mem[0]
    assert none < small < 0.6 * full and chain.fwd.min() > 0 and chain.bwd.min() > 0
