"""The attention oracle itself, on the CPU: gradients against differences, buckets against the library's, the cache against its bound."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

import attn_oracle as ao
import cuts


@pytest.fixture(scope="module")
def borders(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("bucket") / "bucket_query.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", cuts.CSRC, os.path.join(cuts.HERE, "bucket_query.cpp"),
                    "-o", out], check=True)
    lib = C.CDLL(out)
    lib.borders.argtypes = [C.c_int, C.c_int, C.POINTER(C.c_int)]
    lib.borders.restype = None

    def ask(count, far):
        buf = (C.c_int * 128)()
        lib.borders(count, far, buf)
        return list(buf)
    return ask


@pytest.mark.parametrize("count", [2, 3, 4, 7, 16, 31, 32, 64, 127, 128])
@pytest.mark.parametrize("far", [2, 9, 65, 100, 128, 512, 1000, 1024])
def test_borders_are_the_definition(borders, count, far):
    if far <= count // 2:
        pytest.skip("not a bias")
    got = borders(count, far)
    assert got[count - 1:] == [2 ** 31 - 1] * (129 - count)
    want = [ao.bucket(-n, count, far, False) for n in range(far + 1)]
    assert [sum(n >= b for b in got[:count - 1]) for n in range(far + 1)] == want


def test_borders_at_whole_powers(borders):
    """exact = 8, far = 128: every other border is a whole number exactly (16, 32, 64), where logarithms in 32 bits go either way."""
    assert borders(16, 128)[:15] == [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]


def case(seed, causal=False, table=True):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    q, k, v, do = r(2, 3, 4, 5), r(2, 6, 2, 5), r(2, 6, 2, 5), r(2, 3, 4, 5)
    mask = torch.rand(2, 6, generator=gen) < 0.8
    return (q, k, v), do, dict(lens=[6, 4], mask=mask, causal=causal, firsts=[2, 1] if causal else None,
                               table=r(6, 4) if table else None, max_distance=5, two_sided=not causal)


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_are_the_differences(causal):
    (q, k, v), do, how = case(3, causal)
    grads = ao.Case(q, k, v, **how).backward(do)[0]
    for n, name in enumerate(("q", "k", "v", "table")):
        x = dict(q=q, k=k, v=v, table=how["table"])[name]
        for at in range(0, x.numel(), 7):
            sides = []
            for step in (1e-5, -1e-5):
                y = x.clone()
                y.view(-1)[at] += step
                args = dict(q=q, k=k, v=v)
                other = dict(how)
                (other if name == "table" else args)[name] = y
                sides.append(float((ao.Case(**args, **other).forward()[0] * do).sum()))
            assert math.isclose((sides[0] - sides[1]) / 2e-5, float(grads[n].reshape(-1)[at]), rel_tol=1e-6, abs_tol=1e-8), (name, at)


def test_rows_without_keys():
    (q, k, v), do, how = case(5)
    how["lens"] = [0, 6]
    c = ao.Case(q, k, v, **how)
    o, lse, _ = c.forward()
    assert not o[0].any() and bool((lse[0] == -math.inf).all()) and bool(lse[1].isfinite().all())
    dq, dk, dv, _ = c.backward(do)[0]
    assert not dq[0].any() and not dk[0].any() and not dv[0].any()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_cache_values_are_within_half_a_step(dtype):
    x = (torch.randn(50, 24, generator=torch.Generator().manual_seed(1)) * torch.logspace(-3, 3, 50)[:, None]).to(dtype).double()
    c = ao.Cache(64, 24, dtype)
    c.write(x, 5)
    got = c.values()
    assert not got[:5].any() and not got[55:].any()
    steps = torch.tensor([c.step(t // 32) for t in range(5, 55)])[:, None]
    assert bool(((got[5:55] - x).abs() <= steps / 2).all())
    assert torch.equal(got, got.to(dtype).double())  # exact in the type it came from


def test_cache_tokens_that_join_raise_the_step():
    c = ao.Cache(32, 2, torch.bfloat16)
    c.write(torch.tensor([[1.0, -0.5]]).double(), 0)
    assert c.exps[0] - 127 == -6 and c.codes[0].tolist() == [64, -32]
    c.write(torch.tensor([[100.0, 3.0]]).double(), 1)
    assert c.exps[0] - 127 == 0 and c.codes[:2].tolist() == [[1, 0], [100, 3]]  # -0.5 rounds to even
    c.write(torch.tensor([[math.inf, 0.0]]).double(), 2)
    assert c.exps[0] == 255 and bool(c.values().isnan().all())
