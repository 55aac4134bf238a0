"""How many products one launch may hold (csrc/qa_product_plan.h, compiled for the CPU): a launch of 2^32 work-items and more is refused."""
import ctypes as C
import os
import random
import subprocess

import pytest

qa = pytest.importorskip("paper_2208_05631_amd", reason="libqadagrad.so not built")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GROUPS = (256, 256, 256, 512, 512, 256)                          # work-items of a tile, form by form


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("grid") / "product_grid.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_2208_05631_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "product_grid.cpp"), "-o", so], check=True)
    lib = C.CDLL(so)
    lib.most_side_by_side.argtypes, lib.most_side_by_side.restype = [C.c_int64] * 2, C.c_int64
    lib.tiles_of.argtypes, lib.tiles_of.restype = [C.c_int, C.c_int64, C.c_int64, C.c_int64], C.c_int64
    return lib


def test_work_items_of_a_launch(lib):
    rng = random.Random(1)
    shapes = [(1, 16384), (16384, 1), (1, (1 << 20) - 1), (1, 1), (128, 1024)] + [tuple(int(2 ** rng.uniform(0, 20)) for _ in range(2)) for _ in range(2000)]
    for m, n in shapes:
        if m * n >= 1 << 34:
            continue                                             # no card holds it
        most = lib.most_side_by_side(m, n)
        assert most >= 1
        for form, group in enumerate(GROUPS):
            assert lib.tiles_of(form, m, n, min(most, 65535)) * group < 1 << 32, (m, n, form)
    assert lib.most_side_by_side(1, 16384) < 65535 <= lib.most_side_by_side(1, 4096)


def test_a_launchs_share_fits_the_workspace_of_all(lib):
    for m, n in ((1, 16384), (16384, 1), (2, 50000), (40, 9000), (1, (1 << 20) - 1)):
        most = lib.most_side_by_side(m, n)
        for count in (most + 1, 2 * most, 65535):
            if not most < count < 65536:
                continue
            whole = qa.qa_orthogonal_workspace_bytes(qa.Matrices.make(count, m, n), qa.QA_F32)
            for share in (most, count % most):
                assert qa.qa_orthogonal_workspace_bytes(qa.Matrices.make(share, m, n), qa.QA_F32) <= whole
