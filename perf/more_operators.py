"""Performance cases of the attention operators: what a training step of an attention block under a
re-materialization schedule, or a program that runs the trained blocks, calls.

A pass is one use of one operator:

  cross  attention of queries to the keys and values of states of another length, whose heads may be shared by several
         query heads.  ``pass`` fwd: the output.  step: output and row sums, then the gradients of q, k and v from
         what ``keep`` says is kept of the output: 16bit (itself), full (in 32 bits) or none (made again).
  bias   the same with a learned bias by relative position: a table of a number per bucket of distances and head.  The step
         gives the table's gradient too.
  write  tokens written behind those that an 8-bit cache of keys and values holds, and the cache's values after it.
  cache  attention of a few tokens, or of a prompt's next piece, over such a cache.

A key takes part if it lies before its sequence's length, its mask says so and, if ``causal``, it is not behind the query.  A row
without keys has output 0 and log-sum -inf.

The cache keeps a head's tokens in blocks of 32 that share 2^e, the least power of two with max|x| <= 127 * 2^e (e >= -126);
a value is kept as round-half-even(x * 2^-e), a whole number (at most 63 where 64 * 2^e would pass the largest value of x's
type).  A token that joins a block raises e where it has to, and what the block held is rounded to the new step.
"""
import math

import torch

own = False

BLOCK = 32
DTYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f32=torch.float32)
MOST_PRODUCTS = 2 * 16 * 4096 * 4096 * 128  # batch * heads * queries * keys * width of a drawn step, of which a causal one does half
MOST_PAIRS = 2 * 16 * 4096 * 4096           # batch * heads * queries * keys
MOST_CACHE = 16 * 32768 * 8 * 128           # elements of a drawn cache's keys


def _case(op, what, batch, q, k, heads, kv, dim, dtype, **more):
    case = dict(op=op, **{"pass": what}, batch=batch, q=q, k=k, heads=heads, kv=kv, dim=dim, dtype=dtype, ragged=False, mask=False,
                causal=False, at_end=False, keep="none", buckets=0, far=0, two_sided=False, table="")
    case.update(more)
    return case


def listed():
    return [
        # one token of a decoder looks at an encoder's states: all latency
        _case("cross", "fwd", 1, 1, 128, 8, 8, 64, "bf16", name="cross_one_token"),
        # 64 sequences decoded together over states of up to 1500 positions; a batch's idle slot has none
        _case("cross", "fwd", 64, 1, 1500, 16, 16, 64, "f16", ragged=True, name="cross_tokens_64"),
        # a small training step of ragged sizes with shared key heads and positions masked anywhere
        _case("cross", "step", 6, 199, 777, 12, 4, 72, "f16", mask=True, keep="16bit", name="cross_step_ragged"),
        # many queries to few keys, as an image's positions to a short text
        _case("cross", "step", 4, 4096, 77, 10, 10, 64, "bf16", keep="none", name="cross_step_77"),
        # a large training step with shared key heads and padded states
        _case("cross", "step", 4, 2048, 4096, 32, 8, 128, "bf16", ragged=True, keep="16bit", name="cross_step_4096"),
        # an encoder's training step, table in 32 bits, what the backward reads kept in 32 bits
        _case("bias", "step", 16, 512, 512, 12, 12, 64, "bf16", keep="full", buckets=32, far=128, two_sided=True, table="f32",
              name="bias_step_512"),
        # odd sizes, a table of few buckets
        _case("bias", "step", 2, 333, 333, 5, 5, 40, "f16", keep="16bit", buckets=20, far=64, two_sided=True, table="f16",
              name="bias_step_odd"),
        # a decoder's training step over a long sequence
        _case("bias", "step", 2, 4096, 4096, 16, 16, 128, "bf16", causal=True, keep="16bit", buckets=32, far=128, table="bf16",
              name="bias_step_4096"),
        # the next 100 positions of ragged prompts enter a cache of 1024
        _case("write", "write", 8, 100, 1024, 8, 8, 128, "bf16", ragged=True, name="write_100"),
        # one sequence's next token with a bias by position
        _case("cache", "fwd", 1, 1, 1024, 16, 4, 128, "f16", causal=True, at_end=True, buckets=32, far=128, table="f32",
              name="cache_one_token"),
        # a piece of two prompts over what was cached of them before and with them
        _case("cache", "fwd", 2, 256, 4096, 32, 8, 128, "bf16", ragged=True, causal=True, at_end=True, name="cache_prompt_256"),
        # the largest: 16 long sequences decoded together
        _case("cache", "fwd", 16, 1, 32768, 64, 8, 128, "bf16", ragged=True, causal=True, at_end=True, name="cache_tokens_16"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["cross", "cross", "bias", "bias", "write", "cache"])
        kv = spread(1, 16)
        heads = kv * rng.choice([1, 1, 1, 2, 4, 8])
        dim = rng.choice([16, 32, 40, 64, 64, 72, 80, 96, 128, 128, 200, 256, spread(16, 256)])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        batch = spread(1, 64)
        if op in ("cross", "bias"):
            step = rng.random() < 0.7
            q = spread(1, 4096) if step or rng.random() < 0.5 else rng.randint(1, 4)
            k = spread(1, 16384)
            case = _case(op, "step" if step else "fwd", batch, q, k, heads, kv, dim, dtype, ragged=rng.random() < 0.4, mask=rng.random() < 0.3)
            if step:
                case["keep"] = rng.choice(["none", "16bit", "full"])
            if op == "bias":
                case.update(buckets=2 * rng.randint(2, 32), far=spread(64, 512), table=rng.choice(["f32", dtype]),
                            causal=rng.random() < 0.4)
                case["two_sided"] = not case["causal"]
                if not step:
                    case.update(at_end=True, k=max(q, k))
                else:
                    case["k"] = q
            work = case["batch"] * case["heads"] * case["q"] * case["k"]
            if work <= MOST_PAIRS and work * dim <= MOST_PRODUCTS // (1 if step else 4) and batch * case["k"] * heads * dim <= MOST_CACHE // 4:
                return case
        else:
            k = spread(64, 32768)
            if op == "write":
                case = _case(op, "write", batch, min(k, spread(1, 1024)), k, kv, kv, dim, dtype, ragged=rng.random() < 0.6)
                fits = batch * k * kv * dim <= MOST_CACHE // 32
            else:
                case = _case(op, "fwd", batch, min(k, rng.choice([1, 1, 1, 2, spread(1, 512)])), k, heads, kv, dim, dtype,
                             ragged=rng.random() < 0.6, causal=True, at_end=True)
                if rng.random() < 0.4:
                    case.update(buckets=2 * rng.randint(2, 32), far=spread(64, 512), table=rng.choice(["f32", dtype]))
                fits = batch * k * heads * dim <= MOST_CACHE and batch * heads * case["q"] * k <= MOST_PAIRS // 4
            if fits:
                return case


def _lengths(case):
    """Keys of each sequence: all, or between half and all of them, and none in the last of four and more."""
    B, T = case["batch"], case["k"]
    if not case["ragged"]:
        return [T] * B
    return [0 if B >= 4 and b == B - 1 else T - b * T // (2 * B) for b in range(B)]


def _firsts(case):
    """The position of each sequence's first query."""
    return [n - case["q"] if case["at_end"] else 0 for n in _lengths(case)]


def _held(case):
    """A written cache: tokens that each sequence holds before, and those that come in."""
    room = case["k"] - case["q"]
    held = [room if not case["ragged"] else room - b * room // (2 * case["batch"]) for b in range(case["batch"])]
    return held, [case["q"] if not case["ragged"] else case["q"] - b * case["q"] // (2 * case["batch"]) for b in range(case["batch"])]


# ---------------------------------------------------------------- 8-bit blocks and buckets, in elementary operations

def _two_to(e):
    """2^e in 32 bits for whole e in [-126, 127], from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _blocks(x):
    """[batch, tokens, heads, width] as [batch, blocks, 32, heads, width], padded with zeros."""
    B, T, H, D = x.shape
    blocks = (T + BLOCK - 1) // BLOCK
    padded = torch.zeros(B, blocks * BLOCK, H, D, device=x.device, dtype=x.dtype)
    padded[:, :T] = x
    return padded.view(B, blocks, BLOCK, H, D)


def _steps(x):
    """Exponents [batch, blocks, heads] of blocks (32 bits)."""
    part, power = torch.frexp(x.abs().amax(dim=(2, 4)))  # part * 2^power, part in [1/2, 1)
    e = torch.where(part <= 127.0 / 128.0, power - 7, power - 6)
    return torch.where(part > 0, e, torch.full_like(e, -126)).clamp(min=-126)


def _codes(x, e, largest):
    """Whole numbers (32 bits) that blocks are kept as."""
    step = _two_to(e)[:, :, None, :, None]
    most = torch.where(step > largest / 64.0, 63.0, 127.0)
    return torch.minimum(torch.maximum(torch.round(x * _two_to(-e)[:, :, None, :, None]), -most), most)


def _filled(x, largest):
    """codes [batch, heads, tokens, width rounded up to 16] and exponent bytes [batch, heads, blocks] of a cache that holds x."""
    B, T, H, D = x.shape
    blocks = _blocks(x.float())
    e = _steps(blocks)
    codes = torch.zeros(B, H, blocks.shape[1] * BLOCK, (D + 15) // 16 * 16, device=x.device, dtype=torch.int8)
    codes[:, :, :, :D] = _codes(blocks, e, largest).to(torch.int8).view(B, -1, H, D).permute(0, 2, 1, 3)
    return codes, (e + 127).to(torch.uint8).permute(0, 2, 1).contiguous()


def _values(codes, exps, T, D):
    """What a cache stands for (32 bits): [batch, tokens, heads, width]."""
    step = torch.where(exps == 0, torch.zeros_like(exps, dtype=torch.float32), _two_to(exps.to(torch.int32) - 127))
    x = codes[..., :D].float() * step.repeat_interleave(BLOCK, dim=2)[..., None]
    return x[:, :, :T].permute(0, 2, 1, 3)


def _borders(case):
    """The least distance of each bucket but the first, of one side: by comparison of whole numbers, without rounding."""
    count = case["buckets"] // 2 if case["two_sided"] else case["buckets"]
    exact, far = count // 2, case["far"]
    wide = count - exact
    out = list(range(1, exact + 1))
    for i in range(1, wide):
        # the least n with (n / exact)^wide >= (far / exact)^i
        lo, hi = exact, far
        while lo < hi:
            n = (lo + hi) // 2
            if n ** wide * exact ** i >= far ** i * exact ** wide:
                hi = n
            else:
                lo = n + 1
        out.append(lo)
    return out


def _buckets(case, rel):
    """Buckets of relative positions (key less query)."""
    borders = torch.tensor(_borders(case), device=rel.device)
    if case["two_sided"]:
        return torch.bucketize(rel.abs(), borders, right=True) + (rel > 0) * (case["buckets"] // 2)
    return torch.bucketize((-rel).clamp(min=0), borders, right=True)


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    """Queries, keys and values are normal, with a few stronger tokens and columns of the keys, as trained ones are; gradients are small."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    B, Q, T, H, K, D = (case[n] for n in ("batch", "q", "k", "heads", "kv", "dim"))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * scale

    def keys(tokens):
        strong = torch.exp(0.3 * normal(B, tokens, K, 1))
        columns = torch.ones(D, device="cuda")
        columns[torch.rand(D, generator=gen, device="cuda") < 0.02] = 3.0
        return (normal(B, tokens, K, D) * strong * columns).to(dtype), normal(B, tokens, K, D).to(dtype)

    def ints(values):
        return torch.tensor(values, device="cuda", dtype=torch.int32)

    state = dict(case=case)
    if case["op"] == "write":
        held, counts = _held(case)
        state["firsts"], state["counts"] = ints(held), ints(counts)
        kept = [x * (torch.arange(T, device="cuda")[None, :] < state["firsts"][:, None])[:, :, None, None] for x in keys(T)]
        state["k"], state["v"] = keys(Q)
    else:
        state["q"] = normal(B, Q, H, D).to(dtype)
        state["k"], state["v"] = kept = keys(T)
        if case["ragged"]:
            state["lens"] = ints(_lengths(case))
        if case["mask"]:
            state["mask"] = torch.rand(B, T, generator=gen, device="cuda") < 0.8
        if case["at_end"]:
            state["firsts"] = ints(_firsts(case))
        if case["buckets"]:
            state["table"] = normal(case["buckets"], H).to(DTYPES[case["table"]])
        if case["pass"] == "step":
            state["do"] = normal(B, Q, H, D, scale=0.05).to(dtype)
    if case["op"] in ("write", "cache"):
        pairs = [_filled(x, torch.finfo(dtype).max) for x in kept]
        state["codes"], state["exps"] = torch.stack([p[0] for p in pairs]), torch.stack([p[1] for p in pairs])
        if case["op"] == "cache":
            del state["k"], state["v"]
    return state


# ---------------------------------------------------------------- the plain forms (32 bits)

def _live(state):
    """[batch, queries, keys] (or what broadcasts to it): which keys a query sees; and relative positions."""
    case = state["case"]
    at = torch.arange(case["k"], device="cuda", dtype=torch.int32)
    live = torch.ones(1, 1, case["k"], device="cuda", dtype=torch.bool)
    if "lens" in state:
        live = live & (at[None, None, :] < state["lens"][:, None, None])
    if "mask" in state:
        live = live & state["mask"][:, None, :]
    pos = torch.arange(case["q"], device="cuda", dtype=torch.int32)[None, :]
    if "firsts" in state:
        pos = pos + state["firsts"][:, None]
    rel = at[None, None, :] - pos[:, :, None]
    if case["causal"]:
        live = live & (rel <= 0)
    return live, rel


def _plain_write(state):
    case, dtype = state["case"], DTYPES[state["case"]["dtype"]]
    B, T, K, D = (case[n] for n in ("batch", "k", "kv", "dim"))
    firsts, counts = state["firsts"].long()[:, None], state["counts"].long()[:, None]
    at = torch.arange((T + BLOCK - 1) // BLOCK * BLOCK, device="cuda")[None, :]
    old, new = at < firsts, (at >= firsts) & (at < firsts + counts)
    source = (at - firsts).clamp(min=0, max=case["q"] - 1)[:, :, None, None].expand(-1, -1, K, D)
    out = {}
    for i, name in enumerate(("k", "v")):
        before = _values(state["codes"][i], state["exps"][i], at.shape[1], D)
        came = torch.gather(state[name].float(), 1, source)
        e = _steps((came * new[:, :, None, None]).view(B, -1, BLOCK, K, D))
        any_old = old.view(B, -1, BLOCK).any(dim=2)[:, :, None]
        any_new = new.view(B, -1, BLOCK).any(dim=2)[:, :, None]
        e_old = state["exps"][i].permute(0, 2, 1).to(torch.int32) - 127
        e = torch.where(any_new, torch.where(any_old, torch.maximum(e, e_old), e), e_old).clamp(min=-126)
        x = torch.where(old[:, :, None, None], before, came * new[:, :, None, None]).view(B, -1, BLOCK, K, D)
        x = _codes(x, e, torch.finfo(dtype).max) * _two_to(e)[:, :, None, :, None]
        out[name] = x.view(B, -1, K, D)[:, :T].to(dtype)
    return out


def _plain(state):
    case, dtype = state["case"], DTYPES[state["case"]["dtype"]]
    if case["op"] == "write":
        return _plain_write(state)
    B, Q, T, H, K, D = (case[n] for n in ("batch", "q", "k", "heads", "kv", "dim"))
    G = H // K
    if case["op"] == "cache":
        k, v = (_values(state["codes"][i], state["exps"][i], T, D).permute(0, 2, 1, 3) for i in (0, 1))
    else:
        k, v = (state[n].float().permute(0, 2, 1, 3) for n in ("k", "v"))  # [B, K, T, D]
    scale = D ** -0.5

    def grouped(x):  # [B, Q, H, D] as [B, K, G * Q, D]
        return x.float().permute(0, 2, 1, 3).reshape(B, K, G * Q, D)

    def ungrouped(x):
        return x.reshape(B, H, Q, D).permute(0, 2, 1, 3)

    q = grouped(state["q"])
    live, rel = _live(state)
    dead = ~live[:, None]
    if "lens" in state or "mask" in state:  # what lies in dead places counts for nothing
        some = live.any(dim=1)[:, None, :, None]
        k, v = k.masked_fill(~some, 0.0), v.masked_fill(~some, 0.0)
    s = torch.matmul(q, k.transpose(2, 3)).view(B, H, Q, T) * scale
    if case["buckets"]:
        bucket = _buckets(case, rel)
        s = s + state["table"].float().t()[:, bucket].permute(1, 0, 2, 3)
    s = s.masked_fill(dead, -math.inf)
    top = s.amax(dim=3, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    del s
    total = p.sum(dim=3, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(B, K, G * Q, T), v)
    out = dict(o=ungrouped(o).to(dtype))
    if case["pass"] == "step":
        do = grouped(state["do"])
        dv = torch.matmul(p.view(B, K, G * Q, T).transpose(2, 3), do)
        dp = torch.matmul(do, v.transpose(2, 3))
        delta = (do * o).sum(dim=3, keepdim=True)
        ds = p.view(B, K, G * Q, T) * (dp - delta)
        del p, dp
        dq = torch.matmul(ds, k) * scale
        dk = torch.matmul(ds.transpose(2, 3), q) * scale
        if case["keep"] != "none":
            out["lse"] = lse
        out.update(dq=ungrouped(dq).to(dtype), dk=dk.permute(0, 2, 1, 3).to(dtype), dv=dv.permute(0, 2, 1, 3).to(dtype))
        if case["buckets"]:
            # diagonals become columns: rows from the last on, each one place further to the right
            wide = torch.zeros(H, Q, T + Q, device=ds.device)
            wide[:, :, :T] = ds.view(B, H, Q, T).sum(dim=0).flip(1)
            by_distance = wide.view(H, -1)[:, :Q * (T + Q - 1)].view(H, Q, T + Q - 1).sum(dim=1)
            distance = torch.arange(T + Q - 1, device=ds.device) - (Q - 1)
            dtable = torch.zeros(case["buckets"], H, device=ds.device, dtype=torch.float64)
            dtable.index_add_(0, _buckets(case, distance), by_distance.t().double())
            out["dtable"] = dtable.to(state["table"].dtype)
    return out


# ---------------------------------------------------------------- the framework's operators

def _own(state):
    from paper_2307_01236_amd import block

    case = state["case"]
    if case["op"] in ("write", "cache"):
        cache = block.Kv8(state["codes"], state["exps"], (case["batch"], case["k"], case["kv"], case["dim"]), DTYPES[case["dtype"]])
    if case["op"] == "write":
        block.rkb_kv8_write(cache, state["k"], state["v"], state["firsts"], state["counts"])
        k, v = block.rkb_kv8_load(cache)
        return dict(k=k, v=v)
    how = dict(lens=state.get("lens"), mask=state.get("mask"), causal=case["causal"], first=state.get("firsts", 0))
    if case["buckets"]:
        how["bias"] = block.RelBias(state["table"], case["far"], case["two_sided"])
    if case["op"] == "cache":
        return dict(o=block.rkb_attn_fwd(state["q"], cache, **how)[0])
    q, k, v = state["q"], state["k"], state["v"]
    if case["pass"] == "fwd":
        return dict(o=block.rkb_attn_fwd(q, k, v, **how)[0])
    o, kept = block.rkb_attn_fwd(q, k, v, keep=case["keep"], **how)
    out = dict(o=o)
    if case["keep"] != "none":
        out["lse"] = kept[1]
    dq, dk, dv, dtable = block.rkb_attn_bwd(state["do"], q, k, v, kept, **how)
    out.update(dq=dq, dk=dk, dv=dv)
    if case["buckets"]:
        out["dtable"] = dtable
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- the work

def work(case):
    B, Q, T, H, K, D = (case[n] for n in ("batch", "q", "k", "heads", "kv", "dim"))
    if case["op"] == "write":
        held, counts = _held(case)
        # the tokens in, their codes out, and the cache's values: codes in, 16 bits out
        new, all_ = sum(counts) * K * D, B * T * K * D
        return dict(bytes=2.0 * (new * 3 + all_ * 3), flops=2.0 * (5 * new + 2 * all_))
    lens, firsts = _lengths(case), _firsts(case)
    if case["causal"]:
        def seen(n, first):  # sum over queries of how many keys each sees
            full = min(Q, max(0, first + Q - n + 1))  # queries that see all n
            part = Q - full                           # the others see first + 1 .. first + part keys, none below 0
            low = max(first, -1 if part else first)
            steps = max(0, first + part - max(low, 0))
            return full * n + steps * (max(low, 0) + first + part + 1) // 2
        pairs = H * sum(seen(n, f) for n, f in zip(lens, firsts))
    else:
        pairs = H * Q * sum(lens)
    keys, rows = sum(lens) * K * D, B * Q * H * D
    kv_bytes = keys * 2 * 2 if case["op"] != "cache" else keys * 2 + sum(lens) * K * 2 // BLOCK
    moved, products = 2 * rows * 2 + kv_bytes, 2
    if case["pass"] == "step":
        # do in, dq, dk and dv out, row sums out and in again; five products more, and the forward again where nothing is kept
        moved += 2 * rows * 2 + B * T * K * D * 2 * 2 + 8 * B * Q * H
        products += 5 + (2 if case["keep"] == "none" else 0)
    return dict(bytes=float(moved), flops=2.0 * products * pairs * D)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    if case["batch"] * case["heads"] * case["q"] * case["k"] * case["dim"] > MOST_PRODUCTS * 2:
        return None
    state = prepare(case, seed)
    B, Q, T, H, K, D = (case[n] for n in ("batch", "q", "k", "heads", "kv", "dim"))
    largest = float(torch.finfo(DTYPES[case["dtype"]]).max)

    def stored(i):  # the cache's values, [batch, tokens (whole blocks), heads, width], and its exponents
        power = state["exps"][i].double() - 127.0
        wide = power.repeat_interleave(BLOCK, dim=2).unsqueeze(3)
        return (state["codes"][i][..., :D].double() * torch.exp2(wide) * (wide > -127)).transpose(1, 2), power

    if case["op"] == "write":
        held, counts = _held(case)
        out = {}
        for i, name in enumerate(("k", "v")):
            values, power = stored(i)
            values, new = values.clone(), state[name].double()
            for b in range(B):
                if counts[b] == 0:
                    continue
                values[b, held[b]:] = 0.0
                values[b, held[b]:held[b] + counts[b]] = new[b, :counts[b]]
                for block in range(held[b] // BLOCK, (held[b] + counts[b] - 1) // BLOCK + 1):
                    lo, hi = block * BLOCK, block * BLOCK + BLOCK
                    fresh = values[b, max(lo, held[b]):hi].abs().amax(dim=(0, 2)) / 127.0
                    step = torch.exp2(torch.ceil(torch.log2(fresh.clamp(min=2.0 ** -126))))
                    # log2 is rounded: settle the neighbours by comparison, which is exact
                    step = torch.where(fresh > step, step * 2, step)
                    step = torch.where((fresh <= step / 2) & (step > 2.0 ** -126), step / 2, step)
                    if held[b] > lo:
                        step = torch.maximum(step, torch.exp2(power[b, :, block]))
                    step = step[None, :, None]
                    most = torch.where(64.0 * step > largest, 63.0, 127.0).double()
                    values[b, lo:hi] = torch.round(values[b, lo:hi] / step).clamp(-most, most) * step
            out[name] = values[:, :T]
        return out

    if case["op"] == "cache":
        k, v = stored(0)[0][:, :T], stored(1)[0][:, :T]
    else:
        k, v = state["k"].double(), state["v"].double()
    q, scale = state["q"].double(), 1.0 / math.sqrt(D)
    position = torch.arange(T, device="cuda")
    lens, firsts = _lengths(case), _firsts(case)
    step = case["pass"] == "step"
    o, lse = torch.zeros_like(q), torch.full((B, H, Q), -math.inf, device="cuda", dtype=torch.float64)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dtable = torch.zeros(H, max(1, case["buckets"]), device="cuda", dtype=torch.float64)
    for b in range(B):
        sees = (position < lens[b]).unsqueeze(0).expand(Q, T)
        if case["mask"]:
            sees = sees & state["mask"][b].unsqueeze(0)
        ahead = position.unsqueeze(0) - (firsts[b] + torch.arange(Q, device="cuda")).unsqueeze(1)
        if case["causal"]:
            sees = sees & (ahead <= 0)
        some = sees.any(dim=1)
        if case["buckets"]:
            count = case["buckets"] // 2 if case["two_sided"] else case["buckets"]
            near = count // 2
            distance = ahead.abs() if case["two_sided"] else torch.clamp(-ahead, min=0)
            ratio = torch.log(distance.clamp(min=1).double() / near) / math.log(case["far"] / near) * (count - near)
            index = torch.where(distance < near, distance, (near + torch.floor(ratio + 1e-9).long()).clamp(max=count - 1))
            if case["two_sided"]:
                index = torch.where(ahead > 0, index + count, index)
        for h in range(H):
            g = h * K // H
            if not bool(some.any()):
                continue
            kh, vh = k[b, :, g].contiguous(), v[b, :, g].contiguous()
            scores = torch.mm(q[b, :, h].contiguous(), kh.t().contiguous()) * scale
            if case["buckets"]:
                scores = scores + state["table"].double()[:, h][index]
            scores = torch.where(sees, scores, -math.inf)
            lse[b, h] = torch.logsumexp(scores, dim=1)
            p = torch.where(sees, torch.exp(scores - torch.where(some, lse[b, h], 0.0).unsqueeze(1)), 0.0)
            o[b, :, h] = torch.mm(p, vh)
            if step:
                go = state["do"][b, :, h].double().contiguous()
                slope = torch.mm(go, vh.t().contiguous())
                ds = p * (slope - (p * slope).sum(dim=1, keepdim=True))
                dq[b, :, h] = torch.mm(ds, kh) * scale
                dk[b, :, g] += torch.mm(ds.t().contiguous(), q[b, :, h].contiguous()) * scale
                dv[b, :, g] += torch.mm(p.t().contiguous(), go)
                if case["buckets"]:
                    dtable[h] += torch.bincount(index.reshape(-1), weights=ds.reshape(-1), minlength=case["buckets"])
    out = dict(o=o)
    if step:
        if case["keep"] != "none":
            out["lse"] = lse
        out.update(dq=dq, dk=dk, dv=dv)
        if case["buckets"]:
            out["dtable"] = dtable.t().contiguous()
    return out
