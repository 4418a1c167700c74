"""A training step of a chain of gated feed-forward blocks within a memory budget.

Each block is y = x + (act(n Wg^T) * (n Wu^T)) Wd^T with n = layer_norm(x).  The example

  1. measures one block's forwards and backwards on the GPU (times, and memory as torch's allocator
     sees it) for the three options that the block operators offer:
       16bit  keep n, g = n Wg^T, u = n Wu^T and h as 16-bit tensors
       8bit   keep them as 8-bit checkpoints
       none   keep the row statistics; make n, g, u and h again in the backward,
  2. has the solver plan the chain for a budget (rk.Solver), and
  3. runs the plan's steps: forwards that keep nothing, forwards with an option, backwards, and the
     dropping of activations.

Run as a script it prints, for several budgets, the plan's expected time and memory beside the measured ones,
and how far the gradients are from those of the largest budget's plan:

    python examples/train_in_budget.py --layers 12 --tokens 8192 --width 2048 --hidden 5632
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2307_01236_amd import block as bk  # noqa: E402
from paper_2307_01236_amd import rk  # noqa: E402
from paper_2307_01236_amd.chaingen import Chain  # noqa: E402

OPTIONS = ("16bit", "8bit", "none")
NAMES = ("ln_w", "ln_b", "wg", "wu", "wd")


def make_weights(layers: int, width: int, hidden: int, dtype=torch.bfloat16, seed: int = 0, device: str = "cuda"):
    """One dict of weights per block."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale):
        return (torch.randn(*shape, generator=gen, device=device) * scale).to(dtype)

    return [dict(ln_w=1 + normal(width, scale=0.1), ln_b=normal(width, scale=0.1), wg=normal(hidden, width, scale=width ** -0.5),
                 wu=normal(hidden, width, scale=width ** -0.5), wd=normal(width, hidden, scale=(hidden * layers) ** -0.5))
            for _ in range(layers)]


def forward(w, x, option: str | None, act: str = "silu"):
    """(y, what option keeps for the backward); option None keeps nothing (F^0)."""
    n, mean, rstd = bk.rkb_layer_norm_fwd(x, w["ln_w"], w["ln_b"])
    h, gu = bk.rkb_gated_fwd(n, w["wg"], w["wu"], act, keep=option or "none")
    y = torch.addmm(x, h, w["wd"].t())
    if option is None:
        return y, None
    if option == "16bit":
        return y, (mean, rstd, n, gu, h)
    if option == "8bit":
        return y, (mean, rstd, bk.rkb_ckpt8_save(n), gu, bk.rkb_ckpt8_save(h))
    return y, (mean, rstd, None, None, None)


def backward(w, x, dy, kept, option: str, act: str = "silu"):
    """(dx, gradients of the block's weights)"""
    mean, rstd, n, gu, h = kept
    dh = dy @ w["wd"]
    if option == "none":
        n = bk.rkb_layer_norm_fwd(x, w["ln_w"], w["ln_b"])[0]
    dwd = bk.rkb_weight_grad(dy, h) if h is not None else None
    if option == "8bit":
        n = bk.rkb_ckpt8_load(n)
    dn, dwg, dwu, h = bk.rkb_gated_bwd(dh, n, w["wg"], w["wu"], act, gu, want_h=dwd is None)
    if dwd is None:
        dwd = bk.rkb_weight_grad(dy, h)
    dx, dln_w, dln_b = bk.rkb_layer_norm_bwd(dn, x, mean, rstd, w["ln_w"], bias=True)
    return dx.add_(dy), dict(ln_w=dln_w, ln_b=dln_b, wg=dwg, wu=dwu, wd=dwd)


def _timed(call, reps: int = 5):
    """(median microseconds, bytes that stay, bytes beyond those at the peak) of a call, and its result."""
    call()
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = call()
    torch.cuda.synchronize()
    stay = torch.cuda.memory_allocated() - before
    over = torch.cuda.max_memory_allocated() - before - stay
    times = []
    for _ in range(reps):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return float(np.median(times)), stay, over, out


def make_chain(w, x, layers: int, slot: int, options=OPTIONS) -> Chain:
    """The planner's chain for `layers` blocks like w on inputs like x: measured times (microseconds) and sizes
    (slots of `slot` bytes, rounded up)."""
    up = lambda n: -(-max(int(n), 0) // slot)  # noqa: E731
    x_bytes = x.numel() * x.element_size()
    fn_us, _, fn_over, y = _timed(lambda: forward(w, x, None)[0])
    cols = dict(fwd=[], bwd=[], mem=[], tmp_fwd=[], tmp_bwd=[])
    for o in options:
        us, stay, over, (y, kept) = _timed(lambda: forward(w, x, o))
        dy = torch.ones_like(y)
        b_us, b_stay, b_over, out = _timed(lambda: backward(w, x, dy, kept, o))
        for k, v in (("fwd", round(us)), ("bwd", round(b_us)), ("mem", up(stay - x_bytes)), ("tmp_fwd", up(over)),
                     # what the backward leaves (dx, weight gradients until they are stored) and the incoming gradient
                     ("tmp_bwd", up(b_stay + b_over + x_bytes))):
            cols[k].append(v)
        del kept, out, dy
    i32 = lambda a: np.ascontiguousarray(a, dtype=np.int32)  # noqa: E731
    rows = {k: i32([v] * layers) for k, v in cols.items()}
    chain = Chain(L=layers, K=len(options), x=i32([up(x_bytes)] * (layers + 1)), fn_time=i32([round(fn_us)] * layers),
                  fn_tmp=i32([up(fn_over)] * layers), M=0, name="gated_blocks", **rows)
    chain.M = int(chain.x.sum() + chain.mem.max(axis=1).sum() + chain.tmp_fwd.max() + chain.tmp_bwd.max())
    return chain


def run(ops, weights, x0, loss_grad, grads, options=OPTIONS):
    """Run a plan's steps: gradients of every block's weights into `grads` (dicts of tensors like the weights).  Returns
    the gradient of x0."""
    x, kept, dy = {0: x0}, {}, None
    last = len(weights) - 1
    for kind, b, o in ops.tolist():
        if kind == rk.RK_FWD_NOSAVE:
            x[b + 1], _ = forward(weights[b], x[b], None)
        elif kind == rk.RK_FWD_SAVE:
            x[b + 1], kept[b] = forward(weights[b], x[b], options[o])
        elif kind == rk.RK_FREE_X:
            del x[b]
        elif kind == rk.RK_BWD:
            if b == last:
                dy = loss_grad(x[b + 1])
            del x[b + 1]
            dy, new = backward(weights[b], x[b], dy, kept.pop(b), options[o])
            for name in NAMES:
                grads[b][name].copy_(new[name])
            del new
        else:
            raise ValueError(f"unknown step {kind}")
    return dy


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=12)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=5632)
    args = ap.parse_args()
    weights = make_weights(args.layers, args.width, args.hidden)
    grads = [{k: torch.empty_like(v) for k, v in w.items()} for w in weights]
    gen = torch.Generator(device="cuda").manual_seed(1)
    x0 = torch.randn(args.tokens, args.width, generator=gen, device="cuda").bfloat16()
    target = torch.randn(args.tokens, args.width, generator=gen, device="cuda").bfloat16()
    loss_grad = lambda y: (y - target) / args.tokens  # noqa: E731
    slot = x0.numel() * x0.element_size() // 8
    chain = make_chain(weights[0], x0, args.layers, slot)
    for o, name in enumerate(OPTIONS):
        print(f"option {name:6s} forward {chain.fwd[0, o]:6d} us  backward {chain.bwd[0, o]:6d} us  keeps "
              f"{chain.mem[0, o] * slot / 2**20:8.1f} MiB")
    solver = rk.Solver(chain)
    solver.solve()
    curve = solver.tradeoff_curve()
    feasible = np.flatnonzero(curve != rk.RK_INF)
    # the least budget that is as fast as any, the least one at all, and some between
    top, low = int(np.flatnonzero(curve == curve[-1])[0]), int(feasible[0])
    first = None
    for budget in sorted({low, *(low + (top - low) * k // 4 for k in range(1, 4)), top}, reverse=True):
        expect = solver.solve(budget)
        ops, _ = solver.schedule()
        used = [int(((ops[:, 0] == rk.RK_FWD_SAVE) & (ops[:, 2] == o)).sum()) for o in range(len(OPTIONS))]
        run(ops, weights, x0, loss_grad, grads)  # once to warm up
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated() - x0.numel() * x0.element_size()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        run(ops, weights, x0, loss_grad, grads)
        b.record()
        b.synchronize()
        peak = torch.cuda.max_memory_allocated() - before
        flat = torch.cat([g[k].flatten().float() for g in grads for k in NAMES])
        first = flat if first is None else first
        off = float((flat - first).norm() / first.norm())
        print(f"budget {budget * slot / 2**20:9.1f} MiB  expected {expect / 1e3:8.2f} ms  measured {a.elapsed_time(b):8.2f} ms  "
              f"peak {peak / 2**20:9.1f} MiB  blocks " + " ".join(f"{n}:{c}" for n, c in zip(OPTIONS, used)) +
              f"  forwards again {int((ops[:, 0] == rk.RK_FWD_NOSAVE).sum())}  gradients off by {off:.4f}", flush=True)
    solver.close()


if __name__ == "__main__":
    main()
