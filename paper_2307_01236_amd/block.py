"""Python binding of librkblock (include/rk_block.h): argument marshalling only.

Operators of the blocks that a re-materialization schedule runs, on torch tensors of the GPU:
layer norm, checkpoints of activations in 8 bits, the gated feed-forward block and a linear
layer's weight gradient.  Every step runs in the HIP library.  The functions keep the C names;
non-OK return codes raise ``RKBError``, as do tensors that the C call cannot take (off the GPU,
on different devices, of different types, or with columns that are not adjacent).  If
``librkblock.so`` has not been built, loading raises: there is no fallback path.

Leading dimensions count as rows: an [a, b, n] tensor is a matrix of a*b rows and n columns.  Calls are
queued on torch's current stream of the tensors' device and return without waiting; outputs
and workspaces come from torch's allocator, so the calls may be captured into a torch graph.
Tensors that belong to another stream are the caller's to order (wait_stream, record_stream),
as for torch's own operators.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librkblock.so")

RKB_OK, RKB_E_INVAL, RKB_E_NOMEM, RKB_E_DEVICE = 0, -1, -3, -4
RKB_F32, RKB_F16, RKB_BF16 = 0, 1, 2
RKB_SILU, RKB_GELU = 0, 1
RKB_KEEP_NONE, RKB_KEEP_FULL, RKB_KEEP_8BIT, RKB_KEEP_16BIT = 0, 1, 2, 3
RKB_MAX_NORM_COLS = 16384
RKB_MAX_ROWS = 1 << 30
RKB_MAX_COLS = 1 << 24
RKB_GROUP = 32

EXPORTS = ("rkb_layer_norm_fwd", "rkb_layer_norm_bwd_workspace", "rkb_layer_norm_bwd", "rkb_ckpt8_save",
           "rkb_ckpt8_load", "rkb_weight_grad_workspace", "rkb_weight_grad", "rkb_gated_fwd_workspace",
           "rkb_gated_fwd", "rkb_gated_bwd_workspace", "rkb_gated_bwd", "rkb_strerror")

_DTYPE = {torch.float32: RKB_F32, torch.float16: RKB_F16, torch.bfloat16: RKB_BF16}
_ACT = {"silu": RKB_SILU, "gelu": RKB_GELU}
_KEEP = {"none": RKB_KEEP_NONE, "full": RKB_KEEP_FULL, "8bit": RKB_KEEP_8BIT, "16bit": RKB_KEEP_16BIT}

_lib = None


def load():
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


def _refuse(where: str, why: str):
    raise RKBError(RKB_E_INVAL, f"{where} ({why})")


def _check(rc: int, where: str) -> None:
    if rc != RKB_OK:
        raise RKBError(rc, where)


def _matrix(t, where: str, dtype=None, device=None, rows=None, cols=None):
    """(pointer, rows, cols, row stride) of a tensor as a matrix."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(where, "not a tensor of the GPU")
    if dtype is not None and (t.dtype != dtype or t.device != device):
        _refuse(where, "types or devices differ")
    if t.dim() != 2:
        if t.dim() == 0:
            _refuse(where, "no columns")
        try:
            t = t.view(t.numel() // t.shape[-1] if t.shape[-1] else 0, t.shape[-1])
        except RuntimeError:
            _refuse(where, "rows that are not evenly spaced")
    n_rows, n_cols = t.shape
    stride, step = t.stride()
    if step != 1 and n_cols > 1 and n_rows > 0:
        _refuse(where, "columns that are not adjacent")
    if (rows is not None and n_rows != rows) or (cols is not None and n_cols != cols):
        _refuse(where, "sizes do not match")
    return t.data_ptr(), n_rows, n_cols, stride if n_rows > 1 else n_cols


def _vector(t, n: int, where: str, device, dtype):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype != dtype:
        _refuse(where, "types or devices differ")
    if t.numel() != n or not t.is_contiguous():
        _refuse(where, "sizes do not match")
    return t.data_ptr()


def _ckpt(c: Ckpt8, where: str, dtype, device, rows: int, cols: int):
    """(codes, exps) of a checkpoint of a [rows, cols] matrix."""
    ld = -(-cols // RKB_GROUP) * RKB_GROUP
    if c.codes.device != device or c.dtype != dtype:
        _refuse(where, "types or devices differ")
    if (tuple(c.codes.shape) != (rows, ld) or tuple(c.exps.shape) != (rows, ld // RKB_GROUP)
            or not c.codes.is_contiguous() or not c.exps.is_contiguous()):
        _refuse(where, "sizes do not match")
    if c.codes.dtype != torch.int8 or c.exps.dtype != torch.uint8 or c.exps.device != device:
        _refuse(where, "types or devices differ")
    return c.codes.data_ptr(), c.exps.data_ptr()


def _dtype(t, where: str, allowed=_DTYPE):
    if not isinstance(t, torch.Tensor) or t.dtype not in _DTYPE or t.dtype not in allowed:
        _refuse(where, "type")
    return _DTYPE[t.dtype]


_HALF = (torch.float16, torch.bfloat16)


# The current device and a device's current stream, without the objects that torch.cuda wraps
# them in (2 us a call, on calls that take 4).
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else lambda: -1


def _stream(device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _on_its_device(call):
    """Runs a call with its first tensor's device as the current one."""

    @functools.wraps(call)
    def on_device(first, *args, **kw):
        device = getattr(first, "device", None)
        if device is None or device.type != "cuda" or device.index == _current_device():
            return call(first, *args, **kw)
        with torch.cuda.device(device):
            return call(first, *args, **kw)

    return on_device


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name: str, *sizes) -> int:
    """What rkb_<name>_workspace reports, by its arguments."""
    n = C.c_size_t(0)
    _check(getattr(load(), name + "_workspace")(*sizes, C.byref(n)), name)
    return n.value


def _workspace(device, name: str, *sizes):
    """(workspace, pointer, bytes)"""
    n = _workspace_bytes(name, *sizes)
    if not n:
        return None, None, 0
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), n


def _aligned(p: int, stride: int) -> bool:
    return p % 16 == 0 and stride % 8 == 0 and stride <= 1 << 22


def _plain(mats) -> bool:
    """Whether x, wg and wu need no aligned copies (rk_block.h)."""
    xp, xs, wgp, wgs, wup, wus = mats
    return _aligned(xp, xs) and _aligned(wgp, wgs) and _aligned(wup, wus) and wgs == wus


def _weight_type(w, b, x, where: str):
    """The type of a layer norm's weight and bias: x's, or 32-bit (the one's is checked against the other's later)."""
    t = w if w is not None else b
    if t is None:
        return x.dtype
    if t.dtype != x.dtype and t.dtype != torch.float32:
        _refuse(where, "types or devices differ")
    return t.dtype


@_on_its_device
def rkb_layer_norm_fwd(x, weight=None, bias=None, eps: float = 1e-5):
    """(y, mean, rstd): layer norm over the last dimension, and each row's mean and 1 / sqrt(variance + eps)."""
    where = "rkb_layer_norm_fwd"
    dt = _dtype(x, where)
    p, rows, cols, stride = _matrix(x, where)
    device = x.device
    wt = _weight_type(weight, bias, x, where)
    w, b = _vector(weight, cols, where, device, wt), _vector(bias, cols, where, device, wt)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    mean = x.new_empty(x.shape[:-1], dtype=torch.float32)
    rstd = torch.empty_like(mean)
    _check(load().rkb_layer_norm_fwd(dt, _DTYPE[wt], rows, cols, p, stride, w, b, eps, y.data_ptr(), cols, mean.data_ptr(),
                                     rstd.data_ptr(), _stream(device)), where)
    return y, mean, rstd


@_on_its_device
def rkb_layer_norm_bwd(dy, x, mean, rstd, weight=None, bias: bool = False):
    """(dx, dweight, dbias) from dy and what the forward kept: x itself or its Ckpt8, and mean and rstd.
    dweight is None without a weight, dbias unless bias is asked for (it has weight's type, or dy's)."""
    where = "rkb_layer_norm_bwd"
    dt = _dtype(dy, where)
    p, rows, cols, stride = _matrix(dy, where)
    device = dy.device
    wt = _weight_type(weight, None, dy, where)
    w = _vector(weight, cols, where, device, wt)
    m, r = _vector(mean, rows, where, device, torch.float32), _vector(rstd, rows, where, device, torch.float32)
    if m is None or r is None:
        _refuse(where, "no mean or rstd")
    xp, xs, codes, exps = _kept(x, where, dy.dtype, device, rows, cols)
    dx = torch.empty_like(dy, memory_format=torch.contiguous_format)
    dw = torch.empty_like(weight) if weight is not None else None
    db = dy.new_empty(cols, dtype=wt) if bias else None
    ws, ws_p, ws_n = None, None, 0
    if dw is not None or db is not None:
        ws, ws_p, ws_n = _workspace(device, where, dt, rows, cols)
    _check(load().rkb_layer_norm_bwd(dt, _DTYPE[wt], rows, cols, p, stride, xp, xs, codes, exps, m, r, w, dx.data_ptr(), cols,
                                     dw.data_ptr() if dw is not None else None, db.data_ptr() if bias else None, ws_p, ws_n,
                                     _stream(device)), where)
    return dx, dw, db


def _kept(x, where: str, dtype, device, rows: int, cols: int):
    """(pointer, stride, codes, exps) of a matrix that was kept as it was or as a Ckpt8."""
    if isinstance(x, Ckpt8):
        return (None, cols) + _ckpt(x, where, dtype, device, rows, cols)
    p, _, _, stride = _matrix(x, where, dtype, device, rows, cols)
    return p, stride, None, None


def _new_ckpt(like, rows: int, cols: int):
    groups = -(-cols // RKB_GROUP)
    return like.new_empty((rows, groups * RKB_GROUP), dtype=torch.int8), like.new_empty((rows, groups), dtype=torch.uint8)


@_on_its_device
def rkb_ckpt8_save(x) -> Ckpt8:
    """The 8-bit checkpoint of x, in groups of 32 neighbours of the last dimension."""
    where = "rkb_ckpt8_save"
    dt = _dtype(x, where)
    p, rows, cols, stride = _matrix(x, where)
    codes, exps = _new_ckpt(x, rows, cols)
    _check(load().rkb_ckpt8_save(dt, rows, cols, p, stride, codes.data_ptr(), exps.data_ptr(), _stream(x.device)), where)
    return Ckpt8(codes, exps, x.shape, x.dtype)


@_on_its_device
def rkb_ckpt8_load(c: Ckpt8) -> torch.Tensor:
    """The tensor that a checkpoint stands for, of the shape and type it was made from."""
    where = "rkb_ckpt8_load"
    if not isinstance(c, Ckpt8) or not c.codes.is_cuda or c.dtype not in _DTYPE or not c.shape:
        _refuse(where, "not a checkpoint on the GPU")
    device, cols = c.codes.device, c.shape[-1]
    rows = c.shape.numel() // cols if cols else 0
    codes, exps = _ckpt(c, where, c.dtype, device, rows, cols)
    x = c.codes.new_empty(c.shape, dtype=c.dtype)
    _check(load().rkb_ckpt8_load(_DTYPE[c.dtype], rows, cols, codes, exps, x.data_ptr(), cols, _stream(device)), where)
    return x


@_on_its_device
def rkb_weight_grad(dy, x) -> torch.Tensor:
    """dy^T x [n, k], the weight gradient of a linear layer y = x W^T, from dy [..., n] and its input x
    [..., k], kept as it was or as a Ckpt8."""
    where = "rkb_weight_grad"
    dt = _dtype(dy, where, _HALF)
    p, rows, n, stride = _matrix(dy, where)
    if not isinstance(x, (Ckpt8, torch.Tensor)) or not len(x.shape):
        _refuse(where, "not a tensor of the GPU")
    device, k = dy.device, x.shape[-1]
    xp, xs, codes, exps = _kept(x, where, dy.dtype, device, rows, k)
    dw = dy.new_empty((n, k))
    aligned = _aligned(p, stride) and (codes is not None or _aligned(xp, xs))
    ws, ws_p, ws_n = _workspace(device, where, dt, rows, n, k, codes is not None, aligned)
    _check(load().rkb_weight_grad(dt, rows, n, k, p, stride, xp, xs, codes, exps, dw.data_ptr(), k, ws_p, ws_n,
                                  _stream(device)), where)
    return dw


def _gated_args(x, wg, wu, act, where: str):
    if act not in _ACT:
        _refuse(where, "activation")
    dt = _dtype(x, where, _HALF)
    xp, rows, d, xs = _matrix(x, where)
    wgp, f, _, wgs = _matrix(wg, where, x.dtype, x.device, None, d)
    wup, _, _, wus = _matrix(wu, where, x.dtype, x.device, f, d)
    return dt, rows, d, f, (xp, xs, wgp, wgs, wup, wus)


@_on_its_device
def rkb_gated_fwd(x, wg, wu, act: str = "silu", keep: str = "none"):
    """(h, kept): h = act(x wg^T) * (x wu^T) for x [..., d] and wg, wu [f, d]; act is silu or gelu.
    kept is what rkb_gated_bwd takes: None for keep="none", (g, u) as 32-bit tensors for "full", of x's
    type for "16bit", as Ckpt8 for "8bit"."""
    where = "rkb_gated_fwd"
    if keep not in _KEEP:
        _refuse(where, "keep")
    dt, rows, d, f, mats = _gated_args(x, wg, wu, act, where)
    shape = x.shape[:-1] + (f,)
    h = x.new_empty(shape)
    kept, ptrs = None, (None,) * 4
    if keep in ("full", "16bit"):
        kept = tuple(torch.empty_like(h, dtype=torch.float32 if keep == "full" else x.dtype) for _ in range(2))
        ptrs = (kept[0].data_ptr(), kept[1].data_ptr(), None, None)
    elif keep == "8bit":
        kept = tuple(Ckpt8(*_new_ckpt(x, rows, f), shape, torch.float32) for _ in range(2))
        ptrs = tuple(c.codes.data_ptr() for c in kept) + tuple(c.exps.data_ptr() for c in kept)
    ws, ws_p, ws_n = _workspace(x.device, where, dt, rows, d, f, _plain(mats))
    _check(load().rkb_gated_fwd(dt, _ACT[act], _KEEP[keep], rows, d, f, *mats, h.data_ptr(), f, *ptrs, ws_p, ws_n,
                                _stream(x.device)), where)
    return h, kept


@_on_its_device
def rkb_gated_bwd(dh, x, wg, wu, act: str = "silu", kept=None, want_h: bool = False):
    """(dx, dwg, dwu, h) from dh and what rkb_gated_fwd kept; h (None unless want_h) is act(g) * u again, for the
    weight gradient of the layer that follows."""
    where = "rkb_gated_bwd"
    dt, rows, d, f, mats = _gated_args(x, wg, wu, act, where)
    dhp, _, _, dhs = _matrix(dh, where, x.dtype, x.device, rows, f)
    keep, ptrs = RKB_KEEP_NONE, (None,) * 4
    if kept is not None:
        if not isinstance(kept, tuple) or len(kept) != 2:
            _refuse(where, "kept")
        g, u = kept
        if isinstance(g, Ckpt8) and isinstance(u, Ckpt8):
            keep = RKB_KEEP_8BIT
            gp, up = (_ckpt(c, where, torch.float32, x.device, rows, f) for c in (g, u))
            ptrs = (gp[0], up[0], gp[1], up[1])
        else:
            keep = RKB_KEEP_FULL if getattr(g, "dtype", None) == torch.float32 else RKB_KEEP_16BIT
            kind = torch.float32 if keep == RKB_KEEP_FULL else x.dtype
            mats_gu = [_matrix(t, where, kind, x.device, rows, f) for t in (g, u)]
            if any(m[3] != f for m in mats_gu):
                _refuse(where, "g and u are not contiguous")
            ptrs = (mats_gu[0][0], mats_gu[1][0], None, None)
    dx = x.new_empty(x.shape)
    dwg, dwu = x.new_empty((f, d)), x.new_empty((f, d))
    h = x.new_empty(dh.shape) if want_h else None
    ws, ws_p, ws_n = _workspace(x.device, where, dt, keep, rows, d, f, _plain(mats))
    _check(load().rkb_gated_bwd(dt, _ACT[act], keep, rows, d, f, dhp, dhs, *mats, *ptrs, dx.data_ptr(), d, dwg.data_ptr(),
                                dwu.data_ptr(), d, h.data_ptr() if want_h else None, f, ws_p, ws_n, _stream(x.device)), where)
    return dx, dwg, dwu, h
