"""Orthogonalised updates of matrices with few large singular values over a floor of small ones, as gradients have them.

Every step multiplies a small singular value by 3.4, and the noise of its own roundings in that direction too.  What step i adds is some
8 u |X_i|_F (u = 2^-24: three products and their results, as in test_gpu_orthogonal.py), and each later step makes at most 4 times as much of it.
While the floor is low |X_i|_F is that of the few large values.  So after S steps the result is off by at most
    8 u sum_i 4^(S - 1 - i) |X_i|_F,
some 1e-5 of the floor's own part.  That is what the bits of X, A and B are for: one binary16 part leaves some percent."""
import math

import pytest
import torch

import layer_reference as ref

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")

F64 = torch.float64
U = 2.0 ** -24
SHAPES = [(256, 512), (96, 96), (300, 200), (128, 1024), (640, 700)]


def steep(R, C, floor, seed=0):
    """Eight singular values of 1 over `floor`, in binary32."""
    gen = torch.Generator().manual_seed(1000 * R + C + seed)
    n = min(R, C)
    a, _ = torch.linalg.qr(torch.randn(R, n, generator=gen, dtype=F64))
    b, _ = torch.linalg.qr(torch.randn(C, n, generator=gen, dtype=F64))
    s = torch.full((n,), floor, dtype=F64)
    s[:8] = 1.0
    return ((a * s) @ b.t()).float()


def bound(v, steps):
    total, x = 0.0, None
    for i in range(steps):
        x = ref.orthogonal(v, i) if i else v / v.norm()
        total += 4.0 ** (steps - 1 - i) * float(x.norm())
    return 8 * U * total


def rounded(v, bits):
    """To so many leading bits, to nearest."""
    m, e = torch.frexp(v)
    return torch.ldexp(torch.round(m * 2.0 ** bits) * 2.0 ** -bits, e)


@pytest.mark.parametrize("floor", [1e-2, 1e-3])
def test_the_bound_tells_bits_apart(floor):
    """The steps in 64 bits with X, A and B rounded: 22 bits are within the bound, 16 and 11 are not."""
    v = steep(256, 512, floor).to(F64)
    want, most = ref.orthogonal(v, 5), bound(v, 5)
    for bits, within in ((22, True), (16, False), (11, False)):
        x = rounded(v / v.norm(), bits)
        a, b, c = ref.USUAL
        for _ in range(5):
            q = rounded(x @ x.t(), bits)
            x = rounded(a * x + rounded(b * q + c * (q @ q), bits) @ x, bits)
        assert (float((x - want).norm()) <= most) == within, bits


@pytest.mark.gpu
@pytest.mark.parametrize("R,C", SHAPES)
@pytest.mark.parametrize("floor", [1e-2, 1e-3])
def test_small_singular_directions_keep_their_bits(R, C, floor):
    N = 3 if R * C < 100000 else 1
    g = torch.stack([steep(R, C, floor, i) for i in range(N)])
    M = qa.Matrices.make(N, R, C)
    need = qa.qa_orthogonal_workspace_bytes(M, qa.QA_F32)
    ws = torch.full((need // 4,), math.nan, device=DEV) if need else None
    out = torch.full(g.shape, 5.0, device=DEV)
    qa.qa_orthogonalize(M, qa.QA_F32, g.to(DEV), 5, None, out, ws)
    for i in range(N):
        v = g[i].to(F64)
        want = ref.orthogonal(v, 5)
        off = float((out[i].cpu().to(F64) - want).norm())
        assert off <= bound(v, 5) + U * float(want.norm())
