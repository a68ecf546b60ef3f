"""Which rows the attention kernels' blocks take (csrc/attn_span.h, compiled
here with g++): over ascending offsets every row of every sequence once and no
other one, wherever the first sequence starts; over any offsets no row outside
its sequence, as the kernels address the tensors by it."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1903_01814_amd", "csrc")
SRC = os.path.join(ROOT, "tests", "native", "attn_rows.cpp")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rows") / "librows.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror",
                    "-I", CSRC, SRC, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    IP = ctypes.POINTER(ctypes.c_int)
    lib.attn_rows.argtypes = [IP] + [ctypes.c_int] * 4 + [IP]
    lib.attn_rows.restype = ctypes.c_long
    return lib


def rows(lib, start, T, G, TR):
    """Rows outside their sequence, and how often each of the T G is taken."""
    IP = ctypes.POINTER(ctypes.c_int)
    s = np.array(start, np.int32)
    taken = np.zeros(T * G + 1, np.int32)
    bad = lib.attn_rows(s.ctypes.data_as(IP), len(start) - 1, T, G, TR, taken.ctypes.data_as(IP))
    return bad, taken[:T * G]


def check_ascending(lib, start, T, G, TR):
    bad, taken = rows(lib, start, T, G, TR)
    assert bad == 0
    want = np.zeros(T * G, np.int32)
    want[min(max(start[0], 0), T) * G:min(max(start[-1], 0), T) * G] = 1
    assert np.array_equal(taken, want)


@pytest.mark.parametrize("TR", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 7, 16])
@pytest.mark.parametrize("start", [
    [0, 300], [200, 300], [64, 100], [300, 600], [128, 400], [127, 129], [599, 600], [600, 600],
    [1, 1, 1, 2], [500, 500, 501, 600], [-5, 20, 1 << 30], [450, 1 << 30], [0, 0, 0],
    list(range(100, 500)), [333] * 130 + [600]])
def test_late_and_empty_starts(lib, start, G, TR):
    check_ascending(lib, start, 600, G, TR)


@pytest.mark.parametrize("TR", [64, 128])
def test_many_ascending_sets(lib, TR):
    rng = random.Random(TR)
    for _ in range(300):
        T, S, G = rng.randint(1, 3000), rng.choice([1, 2, 5, 63, 64, 65, 300]), rng.randint(1, 9)
        first = rng.choice([0, rng.randint(0, T)])
        cut = sorted(rng.randint(first, T) for _ in range(S))
        check_ascending(lib, [first] + cut, T, G, TR)


@pytest.mark.parametrize("TR", [64, 128])
def test_offsets_in_any_order_stay_inside(lib, TR):
    rng = random.Random(1000 + TR)
    sets = [([0, 1000, 10, 2000], 2000, 4), ([0, 300, 100, 400], 400, 2), ([900, 5], 1000, 3)]
    for _ in range(500):
        T = rng.randint(1, 2000)
        sets.append(([rng.randint(-10, T + 10) for _ in range(rng.choice([2, 3, 9, 66, 200]))], T,
                     rng.randint(1, 9)))
    for start, T, G in sets:
        assert rows(lib, start, T, G, TR)[0] == 0, (start, T, G)
