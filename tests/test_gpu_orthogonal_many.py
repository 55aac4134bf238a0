"""More matrices than one launch holds, long and thin ones."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")

F64 = torch.float64
U = 2.0 ** -24


def test_more_than_a_launch_holds():
    """32800 rows of 16384 (70 GB of workspace): X is g / |g| times what the polynomials make of 1."""
    N, C = 32800, 16384
    M = qa.Matrices.make(N, 1, C)
    gen = torch.Generator(device=DEV).manual_seed(5)
    g = torch.empty(N, 1, C, dtype=torch.bfloat16, device=DEV)
    for part in g.split(4100):
        part.normal_(generator=gen)
    out = torch.full_like(g, 5.0)
    ws = torch.empty(qa.qa_orthogonal_workspace_bytes(M, qa.QA_BF16), dtype=torch.uint8, device=DEV)
    qa.qa_orthogonalize(M, qa.QA_BF16, g, 2, None, out, ws)
    s = 1.0
    for _ in range(2):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    for i in (0, 1, 16383, 32766, 32767, 32768, N - 1):
        v = g[i].to(F64)
        want = v / v.norm() * s
        # s is as near as one step's errors, 8 u, times 1 + 4, which is what the second one makes of the first one's; bfloat16's rounding
        assert float((out[i].to(F64) - want).norm()) <= (5 * 8 * U + 2.0 ** -8) * float(want.norm())
    per = [math.isfinite(float(p.float().abs().sum())) and float((p == 5.0).sum()) == 0 for p in out.split(4100)]
    assert all(per)
