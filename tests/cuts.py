"""How the gated block's products are cut at a size: the library's own choice (csrc/rkb_cut.h), built
for the host."""
import ctypes as C
import os
import subprocess
import tempfile
from collections import namedtuple

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2307_01236_amd", "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

Cut = namedtuple("Cut", "rows bufs splits")  # rows: of a tile
Gated = namedtuple("Gated", "few together fine pair sums dx dw")  # pair: (buffers, splits)

_lib = None


def _load():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as tmp:
            out = os.path.join(tmp, "cut_query.so")
            subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-I", INCLUDE,
                            os.path.join(HERE, "cut_query.cpp"), "-o", out], check=True)
            _lib = C.CDLL(out)
        _lib.gated_cuts.argtypes = [C.c_int64] * 3 + [C.POINTER(C.c_int)]
        _lib.weight_grad_cut.argtypes = [C.c_int64] * 3 + [C.POINTER(C.c_int)]
        _lib.gated_cuts.restype = _lib.weight_grad_cut.restype = None
    return _lib


def gated(rows: int, width: int, hidden: int) -> Gated:
    out = (C.c_int * 14)()
    _load().gated_cuts(rows, width, hidden, out)
    return Gated(bool(out[0]), bool(out[1]), bool(out[2]), (out[3], out[4]), Cut(*out[5:8]), Cut(*out[8:11]), Cut(*out[11:14]))


def weight_grad(rows: int, n: int, k: int) -> Cut:
    out = (C.c_int * 3)()
    _load().weight_grad_cut(rows, n, k, out)
    return Cut(*out)


# Sizes that between them take every tile in every product, whole and in splits, in launches of their own and together.
# Each says what it is there for; the others' columns are what else it takes.
GATED_SIZES = [
    ((1999, 136, 2730), dict(sums=Cut(192, 2, 1), together=True, pair=(4, 3))),
    ((1083, 72, 5510), dict(sums=Cut(256, 2, 1), together=True, pair=(4, 12))),
    ((3000, 1500, 3000), dict(sums=Cut(192, 2, 1), together=True, pair=(4, 1))),
    ((129, 130, 1000), dict(sums=Cut(128, 2, 1), together=True, pair=(2, 8))),
    ((24, 16, 171), dict(few=True, together=True, pair=(2, 1))),
    ((4093, 4085, 4091), dict(sums=Cut(256, 2, 1), together=False, dx=Cut(256, 2, 1), dw=Cut(256, 2, 1))),
    ((3012, 1445, 5265), dict(sums=Cut(256, 2, 1), together=False, dx=Cut(256, 2, 3), dw=Cut(256, 2, 1))),
    ((147, 4285, 7531), dict(sums=Cut(128, 4, 1), together=False, dx=Cut(192, 2, 12), dw=Cut(256, 2, 1))),
    ((7450, 1166, 17), dict(sums=Cut(128, 4, 1), together=False, dx=Cut(192, 2, 1), dw=Cut(128, 2, 24))),
    ((3461, 4579, 259), dict(sums=Cut(128, 4, 1), together=False, dx=Cut(256, 2, 1), dw=Cut(128, 4, 1))),
    ((132, 3951, 7128), dict(together=False, dx=Cut(128, 4, 4), dw=Cut(128, 2, 1))),
    ((3709, 16, 493), dict(sums=Cut(128, 2, 1), together=False, dx=Cut(128, 2, 4), dw=Cut(128, 2, 12))),
    ((5281, 40, 549), dict(together=False, dx=Cut(128, 4, 1), dw=Cut(128, 4, 12))),
    ((2809, 72, 24), dict(together=False, dx=Cut(128, 2, 1), dw=Cut(128, 2, 8))),
]
WEIGHT_GRAD_SIZES = [((272, 24, 17), Cut(128, 2, 1)), ((964, 17, 24), Cut(128, 2, 4)), ((466, 16, 33), Cut(128, 4, 1)),
                     ((28282, 16, 17), Cut(128, 4, 64)), ((333, 1062, 7282), Cut(256, 2, 1)), ((30571, 6830, 129), Cut(256, 2, 8))]
