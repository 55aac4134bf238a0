"""The products' choice of tiles and splits (csrc/qa_product_plan.h, compiled for the CPU)."""
import ctypes as C
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
T256, T192, T128, T128_TWO, T64_TWO, T64_FOUR = range(6)
ALL = 0x3F


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "product_plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_2208_05631_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "product_plan.cpp"), "-o", so], check=True)
    lib = C.CDLL(so)
    lib.product_plan.argtypes = [C.c_uint, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_double, C.c_int64, C.POINTER(C.c_int64)]

    def ask(m, n, steps, count=1, lower=False, allowed=ALL, step=1.0, most=1):
        out = (C.c_int64 * 2)()
        lib.product_plan(allowed, m, n, steps, count, int(lower), step, most, out)
        return tuple(out)
    return ask


def test_measured_sizes_get_the_tiles_that_were_fastest(plan):
    assert plan(4096, 4096, 256, lower=True)[0] == T192
    assert plan(2048, 2048, 512, lower=True)[0] == T128_TWO
    assert plan(1024, 1024, 64, lower=True)[0] in (T64_TWO, T64_FOUR)
    assert plan(4096, 4096, 256)[0] == T256 and plan(8192, 2048, 128)[0] == T256
    assert plan(1024, 128, 8, count=64)[0] in (T128, T64_TWO)
    assert plan(333, 333, 63, count=3, lower=True)[0] in (T64_TWO, T64_FOUR)


def test_only_what_is_allowed_and_no_split_without_steps(plan):
    rng = random.Random(1)
    for _ in range(3000):
        m, n, steps = (int(2 ** rng.uniform(0, 15)) for _ in range(3))
        allowed, most = rng.randrange(1, ALL + 1), rng.choice([1, 1, 7, 64])
        lower = rng.random() < 0.3
        tiles, splits = plan(m, m if lower else n, steps, rng.choice([1, 5, 300]), lower, allowed, rng.choice([0.65, 0.75, 1.0]), most)
        assert allowed >> tiles & 1 and 1 <= splits <= most
        each = -(-steps // splits)
        assert splits == 1 or (each >= 8 and (splits - 1) * each < steps)


def test_long_sums_of_few_tiles_are_split(plan):
    tiles, splits = plan(257, 333, 2049, allowed=1 << T256 | 1 << T128 | 1 << T128_TWO, most=64)
    assert splits >= 8
    assert plan(4096, 8192, 512, allowed=1 << T256 | 1 << T128, most=64)[1] == 1
