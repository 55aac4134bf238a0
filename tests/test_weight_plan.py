"""The weight gradient's choice of tiles and splits (csrc/qa_weight_plan.h, compiled for the CPU): the sizes that the tests take for a
form are sizes that get it, whatever the type, and so is the largest measured case."""
import ctypes as C
import os
import subprocess

import pytest

from weight_grad_shapes import FEW, LARGE, LARGE_SPLIT, SMALL

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "weight_plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_2208_05631_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "weight_plan.cpp"), "-o", so], check=True)
    lib = C.CDLL(so)
    lib.weight_plan.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_int, C.POINTER(C.c_int64)]

    def ask(T, N, K, parts):
        out = (C.c_int64 * 2)()
        lib.weight_plan(T, K, N, parts, out)
        return tuple(out)
    return ask


@pytest.mark.parametrize("parts", [1, 2, 3])
def test_sizes_of_the_tests(plan, parts):
    assert plan(*SMALL, parts) == (128, 1) and plan(*FEW, parts) == (128, 1)
    assert all(plan(*s, parts) == (256, 1) for s in LARGE)
    assert all(plan(*s, parts)[0] == 256 and plan(*s, parts)[1] > 1 for s in LARGE_SPLIT)
    assert plan(16384, 8192, 4096, parts)[0] == 256


@pytest.mark.parametrize("parts", [1, 2, 3])
def test_few_columns_of_dy_have_the_small_tile(plan, parts):
    for T in (1, 100, 16384):
        for N in range(1, 8):
            for K in (1, 4096, 1 << 20):
                tile, splits = plan(T, N, K, parts)
                assert tile == 128 and 1 <= splits <= 64 and (splits == 1 or 64 * splits <= T)
