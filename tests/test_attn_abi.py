"""The attention calls' C ABI on a host without a GPU: structures, workspace sizes, and the refusal of bad arguments before any
device call."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2307_01236_amd import block as bk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "rk_block.h")).read()
P = 1 << 20  # a pointer-like number that is never read: the calls below refuse first


def test_constants_match_header():
    for name in ("RKB_MAX_DIM", "RKB_MAX_BUCKETS", "RKB_MAX_DISTANCE"):
        assert re.search(rf"#define {name} {getattr(bk, name)}\b", HEADER), name
    assert "#define RKB_MAX_TOKENS ((int64_t)1 << 28)" in HEADER and bk.RKB_MAX_TOKENS == 1 << 28


@pytest.mark.parametrize("name,struct", [("rkb_heads", bk.CHeads), ("rkb_attn", bk.CAttn), ("rkb_kv8", bk.CKv8)])
def test_structures_match_header(name, struct):
    body = re.sub(r"/\*.*?\*/", "", re.search(rf"typedef struct {name} {{(.*?)}} {name};", HEADER, re.S).group(1), flags=re.S)
    fields = [f.strip(" *") for line in body.split(";") if line.strip() for f in re.sub(r"^\s*(const )?\w+ ", "", line).split(",")]
    assert fields == [f[0] for f in struct._fields_]


def attn(**more):
    a = dict(dtype=bk.RKB_BF16, causal=0, batch=2, q_rows=3, k_rows=5, heads=4, kv_heads=2, dim=16, scale=0.25, first=0, firsts=None,
             lens=None, mask=None, mask_stride=5, table=None, table_dtype=bk.RKB_BF16, buckets=8, max_distance=16, two_sided=1)
    a.update(more)
    return bk.CAttn(**a)


def heads(rows, n, dim=16, p=P, batch=None, row=None, head=None):
    return bk.CHeads(p, rows * n * dim if batch is None else batch, n * dim if row is None else row, dim if head is None else head)


BAD = [dict(dtype=bk.RKB_F32), dict(dtype=3), dict(batch=-1), dict(q_rows=-1), dict(k_rows=-1), dict(batch=(1 << 28) + 1),
       dict(q_rows=(1 << 28) + 1), dict(k_rows=(1 << 28) + 1), dict(heads=0), dict(kv_heads=0), dict(heads=3), dict(heads=65538, kv_heads=1),
       dict(dim=0), dict(dim=257), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
       dict(first=(1 << 40) + 1), dict(firsts=P + 1), dict(lens=P + 2), dict(mask=P, mask_stride=-1),
       dict(table=P, buckets=7), dict(table=P, buckets=2), dict(table=P, buckets=130), dict(table=P, max_distance=2),
       dict(table=P, max_distance=1025), dict(table=P, table_dtype=bk.RKB_F16), dict(table=P + 1), dict(table=P, two_sided=0, buckets=1),
       dict(batch=1 << 22, q_rows=1 << 10)]


@pytest.mark.parametrize("change", BAD, ids=str)
def test_bad_problems_are_refused(change):
    lib, n, a = bk.load(), C.c_size_t(0), attn(**change)
    q, k = heads(3, 4), heads(5, 2)
    assert lib.rkb_attn_fwd_workspace(a, 0, 1, n) == bk.RKB_E_INVAL
    assert lib.rkb_attn_bwd_workspace(a, 0, 1, n) == bk.RKB_E_INVAL
    assert lib.rkb_attn_fwd(a, q, k, k, None, q, None, None, P, 1 << 30, None) == bk.RKB_E_INVAL
    assert lib.rkb_attn_bwd(a, q, q, k, k, q, None, P, q, k, k, None, P, 1 << 30, None) == bk.RKB_E_INVAL


def fwd_args(**more):
    q, k = heads(3, 4), heads(5, 2)
    args = dict(a=attn(), q=q, k=k, v=heads(5, 2), cache=None, o=heads(3, 4), o32=None, lse=None, ws=P, wsb=1 << 30, stream=None)
    args.update(more)
    return args


@pytest.mark.parametrize("change", [
    dict(a=None), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=heads(3, 4, p=None)), dict(k=heads(5, 2, p=P + 1)),
    dict(v=heads(5, 2, row=-1)), dict(q=heads(3, 4, batch=(1 << 40) + 1)), dict(o=heads(3, 4, head=15)), dict(o=heads(3, 4, row=16)),
    dict(o=heads(3, 4, batch=0)), dict(o32=P + 8), dict(lse=P + 2), dict(cache=bk.CKv8(P, P, 5)),
    dict(k=None, v=None, cache=bk.CKv8(P, P, 4)), dict(k=None, v=None, cache=bk.CKv8(None, P, 5)), dict(k=None, v=None, cache=bk.CKv8(P, None, 5)),
    dict(k=None, v=None, cache=bk.CKv8(P + 8, P, 5)), dict(q=heads(3, 4, row=63), ws=None), dict(q=heads(3, 4, row=63), ws=P + 16),
], ids=lambda c: ",".join(c))
def test_bad_forward_arguments_are_refused(change):
    assert bk.load().rkb_attn_fwd(*fwd_args(**change).values()) == bk.RKB_E_INVAL


def bwd_args(**more):
    q, k = heads(3, 4), heads(5, 2)
    args = dict(a=attn(table=P), d_o=q, q=q, k=k, v=k, o=q, o32=None, lse=P, dq=q, dk=k, dv=k, dtable=P, ws=P, wsb=1 << 30, stream=None)
    args.update(more)
    return args


@pytest.mark.parametrize("change", [
    dict(a=None), dict(d_o=None), dict(q=None), dict(k=None), dict(v=None), dict(dq=None), dict(dk=None), dict(dv=None),
    dict(d_o=heads(3, 4, p=None)), dict(v=heads(5, 2, p=None)), dict(dk=heads(5, 2, p=None)), dict(dv=heads(5, 2, p=None)),
    dict(dq=heads(3, 4, head=8)), dict(dk=heads(5, 2, row=31)), dict(o=None), dict(o32=P), dict(lse=None), dict(lse=P + 1),
    dict(o=heads(3, 4, p=None), o32=P + 4), dict(a=attn()), dict(dtable=P + 1), dict(ws=None), dict(ws=P + 128),
], ids=lambda c: ",".join(c))
def test_bad_backward_arguments_are_refused(change):
    assert bk.load().rkb_attn_bwd(*bwd_args(**change).values()) == bk.RKB_E_INVAL


def test_short_workspaces_are_refused():
    lib, n = bk.load(), C.c_size_t(0)
    a = attn(q_rows=1, k_rows=4096)  # keys in splits
    one = heads(1, 4)
    assert lib.rkb_attn_fwd_workspace(a, 0, 1, n) == bk.RKB_OK and n.value > 0
    long = heads(4096, 2)
    assert lib.rkb_attn_fwd(a, one, long, long, None, one, None, None, P, n.value - 1, None) == bk.RKB_E_NOMEM
    aligned = n.value
    assert lib.rkb_attn_fwd_workspace(a, 0, 0, n) == bk.RKB_OK and n.value > aligned
    args = bwd_args()
    for again in (0, 1):
        assert lib.rkb_attn_bwd_workspace(args["a"], again, 1, n) == bk.RKB_OK and n.value > 0
    kept = bwd_args(o=None, lse=None, wsb=n.value - 1)  # made again
    assert lib.rkb_attn_bwd(*kept.values()) == bk.RKB_E_NOMEM
    assert lib.rkb_attn_fwd_workspace(a, 0, 1, None) == bk.RKB_E_INVAL
    assert lib.rkb_attn_bwd_workspace(a, 0, 1, None) == bk.RKB_E_INVAL


def test_long_caches_fit_and_more_rows_than_a_launch_takes_do_not():
    lib, n = bk.load(), C.c_size_t(0)
    long = dict(batch=256, heads=64, kv_heads=8, q_rows=1, k_rows=1 << 20)
    assert lib.rkb_attn_fwd_workspace(attn(**long), 1, 1, n) == bk.RKB_OK
    assert lib.rkb_attn_bwd_workspace(attn(**{**long, "batch": 512}), 0, 1, n) == bk.RKB_E_INVAL
    for rows, want in ((1 << 28, bk.RKB_OK), ((1 << 28) + 1, bk.RKB_E_INVAL)):
        assert lib.rkb_attn_fwd_workspace(attn(batch=1, heads=1, kv_heads=1, q_rows=rows), 0, 1, n) == want
        assert lib.rkb_attn_bwd_workspace(attn(batch=1, heads=1, kv_heads=1, k_rows=rows), 0, 1, n) == want
    assert lib.rkb_attn_fwd_workspace(attn(batch=2, heads=1, kv_heads=1, q_rows=1 << 28), 0, 1, n) == bk.RKB_E_INVAL


WRITE = dict(dtype=bk.RKB_BF16, batch=2, rows=3, kv_heads=2, dim=16, k=heads(3, 2), v=heads(3, 2), first=0, firsts=None, counts=None,
             cache=bk.CKv8(P, P, 40), stream=None)
LOAD = dict(dtype=bk.RKB_BF16, batch=2, kv_heads=2, dim=16, cache=bk.CKv8(P, P, 40), k=heads(40, 2), v=heads(40, 2), stream=None)


@pytest.mark.parametrize("change", [
    dict(dtype=bk.RKB_F32), dict(batch=-1), dict(rows=-1), dict(kv_heads=0), dict(dim=0), dict(dim=257), dict(k=None), dict(v=None), dict(cache=None),
    dict(k=heads(3, 2, p=None)), dict(v=heads(3, 2, p=P + 1)), dict(k=heads(3, 2, row=-2)), dict(first=1 << 41), dict(firsts=P + 1), dict(counts=P + 3),
    dict(cache=bk.CKv8(P, P, -1)), dict(cache=bk.CKv8(P + 4, P, 40)), dict(cache=bk.CKv8(None, P, 40)), dict(cache=bk.CKv8(P, None, 40)),
    dict(batch=1 << 22, rows=1 << 10), dict(batch=1 << 28, kv_heads=1 << 16, cache=bk.CKv8(P, P, 1 << 28)),
], ids=lambda c: ",".join(c))
def test_bad_writes_are_refused(change):
    assert bk.load().rkb_kv8_write(*{**WRITE, **change}.values()) == bk.RKB_E_INVAL


@pytest.mark.parametrize("change", [
    dict(dtype=bk.RKB_F32), dict(batch=-1), dict(kv_heads=0), dict(dim=0), dict(dim=300), dict(k=None), dict(v=None), dict(cache=None),
    dict(k=heads(40, 2, p=P + 1)), dict(v=heads(40, 2, head=15)), dict(k=heads(40, 2, row=16)), dict(cache=bk.CKv8(P, None, 40)),
    dict(batch=1 << 28, kv_heads=1 << 16, cache=bk.CKv8(P, P, 1 << 28)),
], ids=lambda c: ",".join(c))
def test_bad_loads_are_refused(change):
    assert bk.load().rkb_kv8_load(*{**LOAD, **change}.values()) == bk.RKB_E_INVAL


def test_nothing_to_do_needs_no_pointers():
    lib, none = bk.load(), bk.CHeads(None, 0, 0, 0)
    for change in (dict(batch=0), dict(q_rows=0)):
        assert lib.rkb_attn_fwd(attn(**change), none, heads(5, 2), heads(5, 2), None, none, None, None, None, 0, None) == bk.RKB_OK
    assert lib.rkb_attn_bwd(attn(batch=0), none, none, none, none, none, None, P, none, none, none, None, None, 0, None) == bk.RKB_OK
    assert lib.rkb_kv8_write(*{**WRITE, "rows": 0, "k": none, "v": none}.values()) == bk.RKB_OK
    assert lib.rkb_kv8_write(*{**WRITE, "cache": bk.CKv8(None, None, 0)}.values()) == bk.RKB_OK
    assert lib.rkb_kv8_load(*{**LOAD, "batch": 0, "k": none, "v": none}.values()) == bk.RKB_OK
    assert lib.rkb_kv8_load(*{**LOAD, "k": none, "v": none}.values()) == bk.RKB_OK


def test_the_binding_refuses_host_tensors_and_bad_choices():
    q = torch.zeros(1, 2, 2, 8, dtype=torch.bfloat16)
    cache = bk.Kv8.zeros(1, 40, 2, 8, device="cpu")
    assert cache.codes.shape == (2, 1, 2, 64, 16) and cache.exps.shape == (2, 1, 2, 2) and cache.nbytes() == 4 * 64 * 16 + 8
    for call in (lambda: bk.rkb_attn_fwd(q, q, q), lambda: bk.rkb_attn_fwd(q, cache), lambda: bk.rkb_attn_bwd(q, q, q, q),
                 lambda: bk.rkb_attn_fwd(q, q, q, keep="8bit"), lambda: bk.rkb_attn_fwd(q, q, q, keep="some"),
                 lambda: bk.rkb_kv8_write(cache, q, q), lambda: bk.rkb_kv8_load(cache), lambda: bk.rkb_kv8_write(q, q, q),
                 lambda: bk.rkb_kv8_load(q)):
        with pytest.raises(bk.RKBError) as e:
            call()
        assert e.value.code == bk.RKB_E_INVAL
