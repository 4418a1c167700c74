"""Attention, its bias by relative position and the 8-bit cache (include/rk_block.h) from their definitions in 64
bits, on the CPU, with the error bounds that 32-bit sums and the stated roundings allow.

A bound is the largest error an output may have.  U is the half step of the 16-bit type relative to a value, U32 that of 32
bits.  A 32-bit sum of n terms is off by at most (n + a few) U32 times the sum of the terms' absolute values, whatever its order.
"""
import math
from fractions import Fraction

import torch

U32 = 2.0 ** -24
BLOCK = 32
# half a step relative to a value, half the smallest subnormal
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}


def d(t):
    return t.detach().cpu().double()


def rounding(ref, dtype):
    u, tiny = ROUND[dtype]
    return ref.abs() * u + tiny


# ------------------------------------------------------------------ buckets

def bucket(rel: int, buckets: int, max_distance: int, two_sided: bool) -> int:
    """By the definition, with whole numbers: floor(w ln(n/e) / ln(far/e)) is the most i with (n/e)^w >= (far/e)^i."""
    count = buckets // 2 if two_sided else buckets
    n = abs(rel) if two_sided else max(-rel, 0)
    base = count if two_sided and rel > 0 else 0
    e = count // 2
    if n < e:
        return base + n
    w = count - e
    lhs, ratio = Fraction(n, e) ** w, Fraction(max_distance, e)
    i = 0
    while i < w - 1 and lhs >= ratio ** (i + 1):
        i += 1
    return base + e + i


def bucket_map(q, k, first, buckets, max_distance, two_sided):
    table = {}
    out = torch.empty(q, k, dtype=torch.long)
    for i in range(q):
        for j in range(k):
            rel = j - first - i
            key = max(-max_distance, min(max_distance, rel))  # from max_distance on the last bucket
            if key not in table:
                table[key] = bucket(key, buckets, max_distance, two_sided)
            out[i, j] = table[key]
    return out


# ------------------------------------------------------------------ attention

class Case:
    """One call's arguments in 64 bits: q [B, Q, H, D], k and v [B, T, K, D], lens and firsts lists, mask [B, T] bool."""

    def __init__(self, q, k, v, scale=None, lens=None, mask=None, causal=False, firsts=None, table=None, max_distance=128, two_sided=True):
        self.q, self.k, self.v = d(q), d(k), d(v)
        self.B, self.Q, self.H, self.D = q.shape
        self.T, self.K = k.shape[1], k.shape[2]
        self.scale = float(torch.tensor(scale if scale is not None else self.D ** -0.5, dtype=torch.float32))
        live = torch.ones(self.B, self.Q, self.T, dtype=torch.bool)
        if lens is not None:
            live &= (torch.arange(self.T)[None] < torch.as_tensor(lens)[:, None])[:, None]
        if mask is not None:
            live &= mask.cpu().bool()[:, None]
        self.firsts = [0] * self.B if firsts is None else [firsts] * self.B if isinstance(firsts, int) else list(firsts)
        if causal:
            pos = torch.tensor(self.firsts)[:, None] + torch.arange(self.Q)[None]
            live &= torch.arange(self.T)[None, None] <= pos[:, :, None]
        self.live = live[:, None]
        seen = live.any(1)  # keys that any query sees
        if not causal:
            self.k = torch.where(seen[:, :, None, None], self.k, 0.0)
            self.v = torch.where(seen[:, :, None, None], self.v, 0.0)
        self.table = None
        if table is not None:
            self.table = torch.where(d(table) <= -1e30, -math.inf, d(table))
            self.buckets = torch.stack([bucket_map(self.Q, self.T, f, len(table), max_distance, two_sided) for f in self.firsts])
        G = self.H // self.K
        self.ks, self.vs = (x.repeat_interleave(G, 2).permute(0, 2, 1, 3) for x in (self.k, self.v))  # [B, H, T, D]
        self.qs = self.q.permute(0, 2, 1, 3)

    def scores(self):
        s = self.scale * (self.qs @ self.ks.transpose(2, 3))
        if self.table is not None:
            s = s + self.table[self.buckets].permute(0, 3, 1, 2)
        return torch.where(self.live, s, -math.inf)

    def forward(self):
        """o [B, Q, H, D], lse [B, H, Q], p [B, H, Q, T]"""
        s = self.scores()
        lse = torch.logsumexp(s, 3)
        p = torch.where(self.live & (s > -math.inf), torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[..., None]), 0.0)
        return (p @ self.vs).permute(0, 2, 1, 3), lse, p

    def backward(self, do):
        """dq, dk, dv, dtable (or None), and the terms that the bounds need"""
        o, lse, p = self.forward()
        do = d(do).permute(0, 2, 1, 3)
        dp = do @ self.vs.transpose(2, 3)
        delta = (p * dp).sum(3, keepdim=True)
        ds = p * (dp - delta)
        group = lambda x: x.view(self.B, self.K, -1, self.T, self.D).sum(2).permute(0, 2, 1, 3)  # noqa: E731
        dq = self.scale * (ds @ self.ks).permute(0, 2, 1, 3)
        dk, dv = group(self.scale * (ds.transpose(2, 3) @ self.qs)), group(p.transpose(2, 3) @ do)
        dtable = None if self.table is None else self._by_bucket(ds)
        return (dq, dk, dv, dtable), (p, dp, delta, ds, do, o)

    def _by_bucket(self, x):
        out = torch.zeros(self.table.shape[0], self.H, dtype=torch.float64)
        for b in range(self.B):
            out.index_add_(0, self.buckets[b].reshape(-1), x[b].reshape(self.H, -1).t())
        return out

    # -------------------------------------------------------------- bounds

    def score_error(self):
        """Of a score: a 32-bit sum of exact products, scaled, plus the bias, in steps of log2."""
        size = self.scale * (self.qs.abs() @ self.ks.abs().transpose(2, 3))
        e = (self.D + 16) * U32 * size
        if self.table is not None:
            e = e + 8 * U32 * self.table.nan_to_num(neginf=0.0)[self.buckets].permute(0, 3, 1, 2).abs()
        return torch.where(self.live, e, 0.0)

    def p_error(self, p):
        """Relative error of a probability before its rounding: its score, the row's sum, and the power itself (whose argument is rounded
        too: |s - m| and |lse| are below 2 log2 of anything that counts, 64 covers them)."""
        e = self.score_error()
        # a row's sum is off by its probabilities' errors, weighted by them
        own = e + 80 * U32
        return own + (p * own).sum(3, keepdim=True) + (self.T + 16) * U32

    def forward_bounds(self, dtype, out_dtype=None):
        o, lse, p = self.forward()
        u = ROUND[dtype][0]
        rel = self.p_error(p)
        lost = 2.0 ** -31 if dtype == torch.float16 else 0.0  # what f16 drops of a probability, relative to the row's largest
        e = (p * (rel + u) * (1 + u)) @ self.vs.abs() + (lost + 0 * p) @ self.vs.abs() + (self.T + 16) * U32 * (p @ self.vs.abs())
        e = e.permute(0, 2, 1, 3)
        bound = e + rounding(o, out_dtype or dtype) + U32 * o.abs()
        lse_bound = torch.where(lse > -math.inf, (p * rel).sum(3) + (self.T + 16) * U32 + 4 * U32 * lse.abs(), 0.0) + 1e-30
        return bound, lse_bound, e

    def backward_bounds(self, do, dtype, kept_dtype, table_dtype=None):
        """kept_dtype: what o was kept in (32 bits where it was made again)."""
        (dq, dk, dv, dtable), (p, dp, delta, ds, dos, o) = self.backward(do)
        u, tiny = ROUND[dtype]
        rel = 2 * self.p_error(p)
        e_o = self.forward_bounds(dtype, kept_dtype)[0].permute(0, 2, 1, 3)
        size_dp = dos.abs() @ self.vs.abs().transpose(2, 3)
        e_dp = (self.D + 16) * U32 * size_dp
        spread = dp.abs() + delta.abs() + size_dp
        # delta from the kept o, and corrected by the sum of ds over the row, which is exact but for 32-bit errors
        e_kept = (dos.abs() * e_o).sum(3, keepdim=True) + (self.D + 16) * U32 * (dos.abs() * o.permute(0, 2, 1, 3).abs()).sum(3, keepdim=True)
        e_fixed = (p * (e_dp + (rel + (self.T + 32) * U32) * (spread + e_kept))).sum(3, keepdim=True) \
            + (p * rel).sum(3, keepdim=True) * e_kept + 4 * U32 * delta.abs()
        # f16: ds is scaled up from 2 |do| |v|, and what falls below the range then
        lost = 0.0
        if dtype == torch.float16:
            lost = 2.0 ** -34 * float(2 * dos.norm(dim=3).amax().clamp(min=0) * self.vs.norm(dim=3).amax()) if self.T else 0.0

        def of_ds(e_delta):
            return torch.where(self.live, p * (e_dp + e_delta + (rel + 8 * U32) * (spread + e_delta)), 0.0)

        e1, e2 = of_ds(e_kept), of_ds(e_fixed)
        alive = torch.where(self.live, 1.0, 0.0)
        rounded = lambda e: e + u * (ds.abs() + e) + lost * alive  # noqa: E731
        group = lambda x: x.view(self.B, self.K, -1, self.T, self.D).sum(2).permute(0, 2, 1, 3)  # noqa: E731
        # dq: ds is rounded with the error of delta in it, which is then taken out with rounded probabilities
        dropped = 2.0 ** -38 if dtype == torch.float16 else 0.0
        in_dq = e2 + u * (ds.abs() + e1) + (p * (u + rel) * (1 + u) + dropped * alive) * e_kept + lost * alive
        b_dq = self.scale * (in_dq @ self.ks.abs() + (self.T + 16) * U32 * ((ds.abs() + e1 + p * e_kept) @ self.ks.abs())).permute(0, 2, 1, 3)
        n = self.Q * (self.H // self.K)
        b_dk = group(self.scale * (rounded(e2).transpose(2, 3) @ self.qs.abs() + (n + 16) * U32 * (ds.abs().transpose(2, 3) @ self.qs.abs())))
        b_dv = group((p * (u + rel) * (1 + u) + dropped * alive).transpose(2, 3) @ dos.abs() + (n + 16) * U32 * (p.transpose(2, 3) @ dos.abs()))
        out = [b_dq * 1.01 + rounding(dq, dtype), b_dk * 1.01 + rounding(dk, dtype), b_dv * 1.01 + rounding(dv, dtype), None]
        if dtable is not None:
            out[3] = 1.01 * self._by_bucket(e2 + (self.B * self.Q * self.T + 16) * U32 * ds.abs()) + rounding(dtable, table_dtype)
        return out


# ------------------------------------------------------------------ the cache

class Cache:
    """A head's blocks as the definition has them: codes and exponents in Python's whole numbers, of one sequence and head at a time."""

    def __init__(self, tokens, dim, dtype):
        self.tokens, self.dim, self.largest = tokens, dim, torch.finfo(dtype).max
        self.room = -(-tokens // BLOCK) * BLOCK
        self.codes = torch.zeros(self.room, dim, dtype=torch.float64)
        self.exps = [0] * (self.room // BLOCK)  # stored bytes

    def step(self, n):
        return 0.0 if self.exps[n] == 0 else math.nan if self.exps[n] == 255 else 2.0 ** (self.exps[n] - 127)

    def write(self, x, first):
        """x [rows, dim] (64 bits) from token `first` on."""
        lo, hi = max(first, 0), min(first + len(x), self.tokens)
        if lo >= hi:
            return
        x = x[lo - first:hi - first]
        for n in range(lo // BLOCK, (hi - 1) // BLOCK + 1):
            start = n * BLOCK
            fresh = x[max(start, lo) - lo:min(start + BLOCK, hi) - lo]
            keep = max(lo - start, 0)
            codes = torch.zeros(BLOCK, self.dim, dtype=torch.float64)
            if not bool(torch.isfinite(fresh).all()) or (keep and self.exps[n] == 255):
                self.exps[n] = 255
                self.codes[start + keep:start + BLOCK] = 0
                continue
            top, e = float(fresh.abs().max()), -126
            while top > 127 * 2.0 ** e:
                e += 1
            if keep:
                old = self.exps[n] - 127
                e = max(e, old)
                codes[:keep] = self.codes[start:start + keep] * (2.0 ** (old - e) if self.exps[n] else 0.0)
            at = keep
            codes[at:at + len(fresh)] = fresh / 2.0 ** e
            most = 63.0 if 64 * 2.0 ** e > self.largest else 127.0
            self.codes[start:start + BLOCK] = torch.round(codes).clamp(-most, most)
            self.exps[n] = e + 127

    def values(self):
        steps = torch.tensor([self.step(n) for n in range(len(self.exps))], dtype=torch.float64)
        return (self.codes * steps.repeat_interleave(BLOCK)[:, None])[:self.tokens]


def worst(got, ref, bound):
    """Largest error over its bound (at most 1 when all is well; infinities have to be the same ones; NaN counts as infinite)."""
    if ref.numel() == 0:
        return 0.0
    got = d(got)
    same = got == ref
    r = torch.where(same, 0.0, (got - ref).abs() / bound)
    return float(torch.nan_to_num(r, nan=math.inf).max())
