"""CPU check that the sizes of tokens_sizes.py meet every kernel of the matrix product
with every epilogue: each product's plan is asked for each of them (csrc/gemm_plan.h,
compiled here with g++)."""
import ctypes
import itertools
import os
import subprocess

import pytest

import tokens_sizes as sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1903_01814_amd", "csrc")
SRC = os.path.join(ROOT, "tests", "native", "gemm_plan_query.cpp")

# tiles, and whether a block has a whole one, a part of its contraction, or runs of all
FORMS = {1: [(256, "one"), (256, "run")], 3: []}
for _planes in FORMS:
    FORMS[_planes] += [(t, m) for t in (128, 64) for m in ("one", "split")]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "libgemmplan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC,
                    SRC, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.gemm_plan_query.argtypes = [ctypes.c_int] * 5 + [ctypes.POINTER(ctypes.c_long)]
    return lib


def forms(lib, M, N, K, gated, planes):
    """(tile, how its contraction is divided) of each launch of a product."""
    out = (ctypes.c_long * 18)()
    lib.gemm_plan_query(M, N, K, gated, planes, out)
    return {(out[2 + 8 * i], {0: "run", 1: "one"}.get(out[8 + 8 * i], "split"))
            for i in range(out[0])}


def linear(T, N, K):
    """The products of a projection: tokens, columns, contraction, and whether gated."""
    return {"forward": (T, N, K, 0), "dx": (T, K, N, 0), "dw": (N, K, T, 0)}


def ffn(T, K, F, N):
    W = 2 * ((F + 7) // 8 * 8)
    return {"gated": (T, F, K, 1), "y": (T, N, F, 0), "dg and du": (T, F, N, 0),
            "dx": (T, K, W, 0), "dw1": (W, K, T, 0), "dw2": (N, F, T, 0)}


@pytest.mark.parametrize("products,listed,planes", [
    (linear, sizes.LINEAR_BF16, 1), (linear, sizes.LINEAR_F32, 3), (ffn, sizes.FFN_BF16, 1),
    (ffn, sizes.FFN_F32, 3)], ids=["linear-bf16", "linear-f32", "ffn-bf16", "ffn-f32"])
def test_every_kernel_is_met(lib, products, listed, planes):
    lib.set_cus(256)
    met = set()
    for s in listed:
        for name, (M, N, K, gated) in products(*s).items():
            for form in forms(lib, M, N, K, gated, planes):
                met.add((name, form, N % 8 == 0))
    wanted = set(itertools.product(products(40, 40, 40, 40) if products is ffn else
                                   products(40, 40, 40), FORMS[planes], (True, False)))
    assert wanted <= met, sorted(wanted - met)
