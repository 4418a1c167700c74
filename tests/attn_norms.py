"""How far gradients of attention may be off as a whole (2-norms), beside attn_oracle's bounds of single elements.

A bound of single elements adds up what every rounding may do at worst, all in one direction, and so allows as much as a systematic error of
do . o makes.  As independent errors the same roundings add up as squares.  A rounding is off by at most U = half a step relative to its
value, and by 0.41 U as a root of the mean square (uniform within its step, the value's logarithm uniform within a power of two: U^2 / 3 times
the mean of 1 / m^2 for m in [1, 2), which is 1 / 2).  The bounds below take U for each, 2.4 times that root, so that a norm of many
roundings does not reach them by chance.

`emulate` makes the same gradients with the library's roundings and nothing else, with or without taking what a row's ds add up to out
of do . o, so that a test can show on the CPU which of the two a bound tells apart."""
import torch

import attn_oracle as ao

LIFT = {torch.bfloat16: 0, torch.float16: 7}     # powers of two by which p is raised before it is rounded: forward
P_LIFT = {torch.bfloat16: 0, torch.float16: 14}  # and backward


def case_of(B, Q, T, H, K, D, dtype, k_mean, v_mean, table=False, seed=0):
    """q, k, v, do of the type and the case: keys and values have means, as a trained block's have, and a row's ds add up to 0 beside them."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    q, k, v, do = r(B, Q, H, D).to(dtype), (r(B, T, K, D) + k_mean).to(dtype), (r(B, T, K, D) + v_mean).to(dtype), (0.1 * r(B, Q, H, D)).to(dtype)
    more = dict(table=r(16, H), max_distance=40, two_sided=True) if table else {}
    return (q, k, v, do), more, ao.Case(q, k, v, **more)


def grouped(case, x):  # [B, H, T, D] summed over the heads that share a key head: [B, T, K, D]
    return x.view(case.B, case.K, -1, case.T, case.D).sum(2).permute(0, 2, 1, 3)


def bounds(case, do, dtype, kept_dtype):
    """Largest 2-norms of the errors of dq, dk, dv and dtable (of 32 bits)."""
    grads, (p, dp, delta, ds, dos, o) = case.backward(do)
    u, uk, u32 = ao.ROUND[dtype][0], ao.ROUND[kept_dtype][0], ao.U32
    k2, q2, do2 = (case.ks ** 2).sum(3), (case.qs ** 2).sum(3), (dos ** 2).sum(3)
    many = lambda n: n ** 0.5 + 16  # noqa: E731  n roundings of partial sums, each at most as large as the terms' absolute values together
    # 16 bits.  What a row's ds add up to: of the output's rounded probabilities, and of the output's own rounding
    r2 = u ** 2 * (p ** 2 * dp ** 2).sum(3) + uk ** 2 * (dos ** 2 * o.permute(0, 2, 1, 3) ** 2).sum(3)
    in_ds2, in_pk2 = u ** 2 * ds ** 2, u ** 2 * r2[..., None] * p ** 2
    # 32 bits, of each element by itself: a score, the power's argument (at most 64 where the probability counts), dp
    score = many(case.D) * u32 * case.scale * (case.qs.abs() @ case.ks.abs().transpose(2, 3)) + 64 * u32
    each = p * (score * (dp.abs() + delta.abs()) + many(case.D) * u32 * (dos.abs() @ case.vs.abs().transpose(2, 3)))
    in_ds2 = in_ds2 + each ** 2
    # and of a whole row: do . o as put right (a sum of ds in 32 bits, of elements with those errors), and its probabilities' common factor, which the
    # gradients have as a factor too
    row = many(case.T) * u32 * ds.abs().sum(3) + 4 * u32 * delta[..., 0].abs() + (each ** 2).sum(3).sqrt()
    factor = (case.T + 96) * u32
    norm = lambda x: float(x.sum().sqrt())  # noqa: E731
    n = case.Q * (case.H // case.K)
    dq = case.scale * (norm((in_ds2 + in_pk2) * k2[:, :, None]) + norm((row[..., None] * (p @ case.ks)) ** 2)
                       + many(case.T) * u32 * float((ds.abs() @ case.ks.abs()).norm()))
    dk = case.scale * (norm((in_ds2 + (row[..., None] * p) ** 2) * q2[..., None])
                       + many(n) * u32 * float(grouped(case, ds.abs().transpose(2, 3) @ case.qs.abs()).norm()))
    dv = norm(p ** 2 * (u ** 2 + score ** 2) * do2[..., None]) + many(n) * u32 * float(grouped(case, p.transpose(2, 3) @ dos.abs()).norm())
    out = [b + (u + factor) * float(g.norm()) for b, g in zip((dq, dk, dv), grads)]
    if case.table is None:
        return out + [None]
    of_rows = torch.zeros(case.B, case.H, case.Q, case.table.shape[0], dtype=torch.float64)
    of_rows.scatter_add_(3, case.buckets[:, None].expand(-1, case.H, -1, -1), p)
    return out + [norm(each ** 2) + norm((row[..., None] * of_rows) ** 2) + (u32 + factor) * float(grads[3].norm())
                  + many(case.B * case.Q * case.T) * u32 * float(case._by_bucket(ds.abs()).norm())]


def emulate(case, do, dtype, kept_dtype, corrected=True):
    """dq, dk, dv and dtable with p and ds rounded to dtype where they enter a product, and o to kept_dtype."""
    rounded = lambda x, lift=0: (x * 2.0 ** lift).to(dtype).double() * 2.0 ** -lift  # noqa: E731
    s = case.scores()
    x = torch.exp(s - s.amax(3, keepdim=True))
    total = x.sum(3, keepdim=True)
    o = (rounded(x, LIFT[dtype]) @ case.vs / total).to(kept_dtype).double()
    p, dos = x / total, ao.d(do).permute(0, 2, 1, 3)
    dp = dos @ case.vs.transpose(2, 3)
    delta = (dos * o).sum(3, keepdim=True)
    lift = 0
    if dtype == torch.float16:
        lift = int(12 - torch.ceil(torch.log2(dos.norm(dim=3).max() * case.vs.norm(dim=3).max())))
    ds = p * (dp - delta)
    r = ds.sum(3, keepdim=True) if corrected else 0.0 * delta
    dq = case.scale * (rounded(ds, lift) @ case.ks - r * (rounded(p, P_LIFT[dtype]) @ case.ks))
    ds = p * (dp - delta - r)
    dk = grouped(case, case.scale * (rounded(ds, lift).transpose(2, 3) @ case.qs))
    dv = grouped(case, rounded(p, P_LIFT[dtype]).transpose(2, 3) @ dos)
    out = [g.to(dtype).double() for g in (dq.permute(0, 2, 1, 3), dk, dv)]
    return out + [None if case.table is None else case._by_bucket(ds).float().double()]


def errors(case, do, got):
    """2-norms of the errors of dq, dk, dv and dtable."""
    return [None if g is None else float((ao.d(g) - r).norm()) for g, r in zip(got, case.backward(do)[0])]


# B, Q, T, heads, key heads, width, a bias.  Keys in splits: 600 and 1500 of few sequences; queries in splits: 700.
SHAPES = {"short": (2, 100, 16, 4, 2, 64, False), "two_tiles": (2, 100, 150, 4, 4, 64, True), "key_splits": (1, 100, 600, 4, 2, 64, True),
          "more_key_splits": (1, 70, 1500, 2, 1, 128, False), "query_splits": (1, 700, 150, 2, 2, 40, True), "wide": (1, 100, 600, 2, 1, 256, False)}
