"""CPU checks of how matrix products are divided among blocks (csrc/gemm_plan.h,
compiled here with g++): the parts cover every row once, tiles cover every column,
splits and runs cover every step of the contraction once, and the split sums fit
the workspace that the plan asks for."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1903_01814_amd", "csrc")
SRC = os.path.join(ROOT, "tests", "native", "gemm_plan_query.cpp")

KSTEP = {(1, 256): 32, (1, 128): 32, (1, 64): 64, (3, 128): 32, (3, 64): 32}


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "libgemmplan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC,
                    SRC, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.gemm_plan_query.argtypes = [ctypes.c_int] * 5 + [ctypes.POINTER(ctypes.c_long)]
    return lib


def plan(lib, M, N, K, gated, planes):
    out = (ctypes.c_long * 18)()
    lib.gemm_plan_query(M, N, K, gated, planes, out)
    names = ("tile", "first", "rows", "mt", "nt", "steps", "splits", "per")
    return out[1], [dict(zip(names, out[2 + 8 * i:10 + 8 * i])) for i in range(out[0])]


def check(lib, M, N, K, gated, planes, cus):
    nbytes, parts = plan(lib, M, N, K, gated, planes)
    assert 1 <= len(parts) <= 2
    row = 0
    for p in parts:
        assert p["first"] == row and p["rows"] >= 1
        row += p["rows"]
        tile = p["tile"]
        cols = tile // 2 if gated and tile > 64 else tile
        assert (p["mt"] - 1) * tile < p["rows"] <= p["mt"] * tile
        assert (p["nt"] - 1) * cols < N <= p["nt"] * cols
        ks = KSTEP[planes, tile]
        assert (p["steps"] - 1) * ks < K <= p["steps"] * ks
        if p["splits"] == 0:  # runs
            assert tile == 256 and planes == 1
            tiles = p["mt"] * p["nt"]
            everything = tiles * p["steps"]
            assert everything >= cus  # no block without a step
            assert nbytes >= (tiles + cus) * 256 * 256 * 4
            bounds = [b * everything // cus for b in range(cus + 1)]
            seen = set()
            for b in range(cus):
                at = bounds[b]
                while at < bounds[b + 1]:
                    t, first = divmod(at, p["steps"])
                    n = min(p["steps"] - first, bounds[b + 1] - at)
                    # the place of a run's sums, and who the join thinks wrote them
                    assert t + b < tiles + cus and t + b not in seen
                    seen.add(t + b)
                    u = t * p["steps"]
                    b0 = ((u + 1) * cus - 1) // everything
                    b1 = ((u + p["steps"]) * cus - 1) // everything
                    assert b0 <= b <= b1 and (b0 == b1) == (n == p["steps"])
                    if first == 0:
                        assert b == b0
                    if first + n == p["steps"]:
                        assert b == b1
                    at += n
        else:
            assert (p["splits"] - 1) * p["per"] < p["steps"] <= p["splits"] * p["per"]
            if p["splits"] > 1:
                width = (N + 7) // 8 * 8 * (2 if gated else 1)
                assert nbytes >= p["splits"] * p["rows"] * width * 4
    assert row == M


@pytest.mark.parametrize("cus", [256, 304, 64])
@pytest.mark.parametrize("planes", [1, 3])
@pytest.mark.parametrize("gated", [0, 1])
def test_plans_cover(lib, gated, planes, cus):
    rng = random.Random(gated * 2 + planes + cus)
    lib.set_cus(cus)
    sizes = lambda: max(1, int(2 ** rng.uniform(0, 14.5)) + rng.choice([-1, 0, 0, 1]))  # noqa: E731
    for _ in range(300):
        check(lib, sizes(), sizes(), sizes(), gated, planes, cus)
    for M, N, K in [(16432, 2048, 5464), (10928, 2048, 16432), (1024, 1024, 51200), (1, 1, 1),
                    (1 << 20, 8, 8), (8, 1 << 20, 40), (513, 1 << 14, 1 << 14)]:
        check(lib, M, N, K, gated, planes, cus)
    lib.set_cus(256)
