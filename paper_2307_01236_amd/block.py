"""Python binding of librkblock (include/rk_block.h): argument marshalling only.

Operators of the blocks that a re-materialization schedule runs, on torch tensors of the GPU:
layer norm, checkpoints of activations in 8 bits, the gated feed-forward block, a linear
layer's weight gradient, and attention (with a bias by relative position, and over a cache of keys and values in 8 bits).  Every step runs in the HIP library; the marshalling itself is native
(csrc/rkb_bind.cpp), because the smallest calls take no longer than marshalling in Python
does.  The functions keep the C names; non-OK return codes raise ``RKBError``, as do tensors that
the C call cannot take (off the GPU, on different devices, of different types, or with columns
that are not adjacent).  If the libraries have not been built, the first call raises: there is no
fallback path.

Leading dimensions count as rows: an [a, b, n] tensor is a matrix of a*b rows and n columns.  Calls are
queued on torch's current stream of the tensors' device and return without waiting; outputs
and workspaces come from torch's allocator, so the calls may be captured into a torch graph.
Tensors that belong to another stream are the caller's to order (wait_stream, record_stream),
as for torch's own operators.  No call takes part in autograd.
"""
from __future__ import annotations

import ctypes as C
import importlib
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librkblock.so")
BIND_PATH = os.path.join(HERE, "_rkblock.so")

RKB_OK, RKB_E_INVAL, RKB_E_NOMEM, RKB_E_DEVICE = 0, -1, -3, -4
RKB_F32, RKB_F16, RKB_BF16 = 0, 1, 2
RKB_SILU, RKB_GELU = 0, 1
RKB_KEEP_NONE, RKB_KEEP_FULL, RKB_KEEP_8BIT, RKB_KEEP_16BIT = 0, 1, 2, 3
RKB_MAX_NORM_COLS = 16384
RKB_MAX_ROWS = 1 << 30
RKB_MAX_COLS = 1 << 24
RKB_GROUP = 32
RKB_MAX_DIM = 256
RKB_MAX_TOKENS = 1 << 28
RKB_MAX_BUCKETS = 128
RKB_MAX_DISTANCE = 1024

EXPORTS = ("rkb_layer_norm_fwd", "rkb_layer_norm_bwd_workspace", "rkb_layer_norm_bwd", "rkb_ckpt8_save",
           "rkb_ckpt8_load", "rkb_weight_grad_workspace", "rkb_weight_grad", "rkb_gated_fwd_workspace",
           "rkb_gated_fwd", "rkb_gated_bwd_workspace", "rkb_gated_bwd", "rkb_kv8_write", "rkb_kv8_load",
           "rkb_attn_fwd_workspace", "rkb_attn_fwd", "rkb_attn_bwd_workspace", "rkb_attn_bwd", "rkb_strerror")

_ACT = {"silu": RKB_SILU, "gelu": RKB_GELU}
_KEEP = {"none": RKB_KEEP_NONE, "full": RKB_KEEP_FULL, "8bit": RKB_KEEP_8BIT, "16bit": RKB_KEEP_16BIT}

_lib = _bind = None


class CHeads(C.Structure):
    """rkb_heads: a [batch, rows, heads, dim] tensor's pointer and strides in elements."""

    _fields_ = [("p", C.c_void_p), ("batch", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


class CAttn(C.Structure):
    """rkb_attn: what a call attends to what."""

    _fields_ = [("dtype", C.c_int), ("causal", C.c_int), ("batch", C.c_int64), ("q_rows", C.c_int64), ("k_rows", C.c_int64),
                ("heads", C.c_int64), ("kv_heads", C.c_int64), ("dim", C.c_int64), ("scale", C.c_float), ("first", C.c_int64),
                ("firsts", C.c_void_p), ("lens", C.c_void_p), ("mask", C.c_void_p), ("mask_stride", C.c_int64),
                ("table", C.c_void_p), ("table_dtype", C.c_int), ("buckets", C.c_int), ("max_distance", C.c_int),
                ("two_sided", C.c_int)]


class CKv8(C.Structure):
    """rkb_kv8: a cache's codes and exps, and the most tokens of a sequence."""

    _fields_ = [("codes", C.c_void_p), ("exps", C.c_void_p), ("tokens", C.c_int64)]


def load():
    """The C library itself, for callers with pointers of their own."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2307_01236_amd.build.build()")
        # torch is imported above: the library binds to torch's HIP runtime, so that memory and
        # streams are shared
        lib = C.CDLL(LIB_PATH)
        i, l, p, sz = C.c_int, C.c_int64, C.c_void_p, C.c_size_t
        szp = C.POINTER(sz)
        lib.rkb_layer_norm_fwd.argtypes = [i, i, l, l, p, l, p, p, C.c_float, p, l, p, p, p]
        lib.rkb_layer_norm_bwd_workspace.argtypes = [i, l, l, szp]
        lib.rkb_layer_norm_bwd.argtypes = [i, i, l, l, p, l, p, l, p, p, p, p, p, p, l, p, p, p, sz, p]
        lib.rkb_ckpt8_save.argtypes = [i, l, l, p, l, p, p, p]
        lib.rkb_ckpt8_load.argtypes = [i, l, l, p, p, p, l, p]
        lib.rkb_weight_grad_workspace.argtypes = [i, l, l, l, i, i, szp]
        lib.rkb_weight_grad.argtypes = [i, l, l, l, p, l, p, l, p, p, p, l, p, sz, p]
        lib.rkb_gated_fwd_workspace.argtypes = [i, l, l, l, i, szp]
        lib.rkb_gated_fwd.argtypes = [i, i, i, l, l, l] + [p, l] * 4 + [p] * 4 + [p, sz, p]
        lib.rkb_gated_bwd_workspace.argtypes = [i, i, l, l, l, i, szp]
        lib.rkb_gated_bwd.argtypes = [i, i, i, l, l, l] + [p, l] * 4 + [p] * 4 + [p, l, p, p, l, p, l, p, sz, p]
        heads, attn, kv8 = C.POINTER(CHeads), C.POINTER(CAttn), C.POINTER(CKv8)
        lib.rkb_kv8_write.argtypes = [i, l, l, l, l, heads, heads, l, p, p, kv8, p]
        lib.rkb_kv8_load.argtypes = [i, l, l, l, kv8, heads, heads, p]
        lib.rkb_attn_fwd_workspace.argtypes = [attn, i, i, szp]
        lib.rkb_attn_fwd.argtypes = [attn, heads, heads, heads, kv8, heads, p, p, p, sz, p]
        lib.rkb_attn_bwd_workspace.argtypes = [attn, i, i, szp]
        lib.rkb_attn_bwd.argtypes = [attn] + [heads] * 5 + [p, p] + [heads] * 3 + [p, p, sz, p]
        lib.rkb_strerror.argtypes = [i]
        lib.rkb_strerror.restype = C.c_char_p
        for n in EXPORTS:
            if n != "rkb_strerror":
                getattr(lib, n).restype = C.c_int
        _lib = lib
    return _lib


def rkb_strerror(code: int) -> str:
    return load().rkb_strerror(int(code)).decode()


class RKBError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {rkb_strerror(code)} ({code})")


class Ckpt8:
    """An 8-bit checkpoint: codes [rows, columns rounded up to 32] (int8), one exponent byte for each 32
    columns, and the shape and type of the tensor it was made from."""

    __slots__ = ("codes", "exps", "shape", "dtype")

    def __init__(self, codes, exps, shape, dtype):
        self.codes, self.exps, self.shape, self.dtype = codes, exps, torch.Size(shape), dtype

    @property
    def device(self):
        return self.codes.device

    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()


class Kv8:
    """A cache of keys and values in 8 bits: codes [2, batch, heads, tokens rounded up to 32, width rounded up to 16] (int8; keys, then
    values), one exponent byte for each 32 tokens of a head, the shape (batch, tokens, heads, width) and the 16-bit type of what it holds."""

    __slots__ = ("codes", "exps", "shape", "dtype")

    def __init__(self, codes, exps, shape, dtype):
        self.codes, self.exps, self.shape, self.dtype = codes, exps, torch.Size(shape), dtype

    @classmethod
    def zeros(cls, batch: int, tokens: int, heads: int, dim: int, dtype=torch.bfloat16, device="cuda") -> "Kv8":
        """An empty cache, for up to `tokens` tokens of each sequence."""
        blocks, ld = -(-tokens // RKB_GROUP), -(-dim // 16) * 16
        return cls(torch.zeros(2, batch, heads, blocks * RKB_GROUP, ld, dtype=torch.int8, device=device),
                   torch.zeros(2, batch, heads, blocks, dtype=torch.uint8, device=device), (batch, tokens, heads, dim), dtype)

    @property
    def device(self):
        return self.codes.device

    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()


class RelBias:
    """A learned bias by relative position: table [buckets, heads] (of the queries' type or 32 bits).  two_sided: half of the buckets for
    keys up to the query and half for those behind it, else all for those up to it.  Half of a side's buckets are
    one distance each, the others grow with its logarithm up to max_distance."""

    __slots__ = ("table", "max_distance", "two_sided")

    def __init__(self, table, max_distance: int = 128, two_sided: bool = True):
        self.table, self.max_distance, self.two_sided = table, max_distance, two_sided


def _native():
    global _bind
    if _bind is None:
        load()
        if not os.path.exists(BIND_PATH):
            raise ImportError(f"{BIND_PATH} is missing: build it with paper_2307_01236_amd.build.build()")
        bind = importlib.import_module("paper_2307_01236_amd._rkblock")
        bind.init(RKBError, Ckpt8, (torch.float32, torch.float16, torch.bfloat16), Kv8, RelBias)
        _bind = bind
    return _bind


def _choice(names: dict, name, where: str, what: str) -> int:
    if name not in names:
        raise RKBError(RKB_E_INVAL, f"{where} ({what})")
    return names[name]


def rkb_layer_norm_fwd(x, weight=None, bias=None, eps: float = 1e-5):
    """(y, mean, rstd): layer norm over the last dimension, and each row's mean and 1 / sqrt(variance + eps).
    x is of 32 or 16 bits, weight and bias of x's type or of 32 bits; y has x's type, mean and rstd 32 bits."""
    return _native().layer_norm_fwd(x, weight, bias, eps)


def rkb_layer_norm_bwd(dy, x, mean, rstd, weight=None, bias: bool = False):
    """(dx, dweight, dbias) from dy and what the forward kept: x itself or its Ckpt8, and mean and rstd.
    dweight is None without a weight, dbias unless bias is asked for (it has weight's type, or dy's)."""
    return _native().layer_norm_bwd(dy, x, mean, rstd, weight, bias)


def rkb_ckpt8_save(x) -> Ckpt8:
    """The 8-bit checkpoint of x, in groups of 32 neighbours of the last dimension."""
    return _native().ckpt8_save(x)


def rkb_ckpt8_load(c: Ckpt8) -> torch.Tensor:
    """The tensor that a checkpoint stands for, of the shape and type it was made from."""
    return _native().ckpt8_load(c)


def rkb_weight_grad(dy, x) -> torch.Tensor:
    """dy^T x [n, k], the weight gradient of a linear layer y = x W^T, from dy [..., n] and its input x
    [..., k], kept as it was or as a Ckpt8 (loaded whole into a workspace).  16-bit types."""
    return _native().weight_grad(dy, x)


def rkb_gated_fwd(x, wg, wu, act: str = "silu", keep: str = "none"):
    """(h, kept): h = act(x wg^T) * (x wu^T) for x [..., d] and wg, wu [f, d] of a 16-bit type; act is silu or gelu.
    kept is what rkb_gated_bwd takes: None for keep="none", (g, u) as 32-bit tensors for "full", of x's
    type for "16bit", as Ckpt8 for "8bit".  h is the same bits whatever is kept."""
    where = "rkb_gated_fwd"
    return _native().gated_fwd(x, wg, wu, _choice(_ACT, act, where, "activation"), _choice(_KEEP, keep, where, "keep"))


def rkb_gated_bwd(dh, x, wg, wu, act: str = "silu", kept=None, want_h: bool = False):
    """(dx, dwg, dwu, h) from dh and what rkb_gated_fwd kept; h (None unless want_h) is act(g) * u again, for the
    weight gradient of the layer that follows.  The gradients of g and u are rounded to x's type on the way."""
    return _native().gated_bwd(dh, x, wg, wu, _choice(_ACT, act, "rkb_gated_bwd", "activation"), kept, want_h)


def rkb_attn_fwd(q, k, v=None, scale: float | None = None, lens=None, mask=None, causal: bool = False, first=0, bias=None,
                 keep: str = "none"):
    """(o, kept): attention of q [batch, queries, heads, width] to k and v [batch, keys, key heads, width], or to a Kv8 given as k.
    Types are 16-bit, heads a multiple of the key heads, which neighbouring heads share, and scale width ** -0.5 unless given.

    lens (int32 [batch]) is each sequence's number of keys, mask ([batch, keys], bool) says which keys take part, and with causal a
    query sees the keys up to its own position: first + its row; first is an int or an int32 tensor [batch].  bias is
    a RelBias.  A query that sees no key has o = 0 (and log-sum -inf).  kept is what rkb_attn_bwd takes: None for
    keep="none", (o, lse) for "16bit", and for "full" o in 32 bits in its place; lse is [batch, heads, queries] in 32 bits."""
    where = "rkb_attn_fwd"
    kind = _choice(_KEEP, keep, where, "keep")
    if kind == RKB_KEEP_8BIT:
        raise RKBError(RKB_E_INVAL, f"{where} (keep)")
    return _native().attn_fwd(q, k, v, scale, lens, mask, causal, first, bias, kind)


def rkb_attn_bwd(do, q, k, v, kept=None, scale: float | None = None, lens=None, mask=None, causal: bool = False, first=0,
                 bias=None):
    """(dq, dk, dv, dtable) from do and what rkb_attn_fwd kept for the same arguments (None: the forward's output is made again); dtable
    is the gradient of the bias's table, None without one.  Sums are in 32 bits and in a fixed order; probabilities and the scores'
    gradients are rounded to q's type on their way into the products."""
    return _native().attn_bwd(do, q, k, v, kept, scale, lens, mask, causal, first, bias)


def rkb_kv8_write(cache: Kv8, k, v, first=0, counts=None) -> None:
    """Writes k and v [batch, rows, key heads, width] into a cache from token `first` of each sequence on (an int, or an int32 tensor
    [batch]); counts (int32 [batch]) is each sequence's number of rows, all unless given.  Tokens before stay, rounded again
    where a block of 32 needs a larger step; rows outside the cache are dropped.  A call takes up to 2^22 blocks of all sequences and key
    heads (rk_block.h): with 8 key heads, a prompt of 4096 tokens for 4064 sequences at once."""
    _native().kv8_write(cache, k, v, first, counts)


def rkb_kv8_load(cache: Kv8):
    """(k, v): what a cache stands for, [batch, tokens, key heads, width] of its type."""
    return _native().kv8_load(cache)
