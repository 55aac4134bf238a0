"""The orthogonalised update and its step against the formulas in 64 bits.

Tolerances.  u = 2^-24.  Numbers are held in 22 bits and a sign (2^-23 relative, and 2^-35 = 2^-25 / 2^10 absolute), products leave out
2^-22 of their terms, sums of k terms are rounded 3 k / 16 + 16 times.  For ONE step, with |.| taken element by element and
T = |X| + |b| |X||X^T||X| ... (the terms of each factor), an element is off by at most the sum over its factors of these errors times the
product of the others' magnitudes.  Over several steps errors grow with the polynomial's slope, which is at most 4 on [0, 1.2]
(3.44 at 0, 3.9 at 1.2), and so does the whole map's, in the Frobenius norm: after S steps by (4^S - 1) / 3 = 341 for S = 5 of what one step
adds, which is some 8 u |X|_F (independent roundings of three products and their results)."""
import math
import zlib

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")

F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U = 2.0 ** -24


def code_of(t):
    return {"f32": qa.QA_F32, "bf16": qa.QA_BF16, "f16": qa.QA_F16}[t]


def gen_of(*what):
    return torch.Generator().manual_seed(zlib.crc32(repr(what).encode()))


def matrices_of(gen, N, R, C, t, pad=0, lead=0, scale=1.0):
    v = (torch.randn(N, R, C, generator=gen) * scale).to(TYPES[t])
    flat = torch.full((lead + N * R * (C + pad) + 8,), 7.0, dtype=TYPES[t], device=DEV)
    d = flat[lead:lead + N * R * (C + pad)].view(N, R, C + pad)
    d[:, :, :C] = v.to(DEV)
    return v.to(F64), d


def room(M, t):
    """Filled with NaN: nothing that a call reads there may be older than the call."""
    need = qa.qa_orthogonal_workspace_bytes(M, code_of(t))
    return torch.full((need // 4,), math.nan, device=DEV) if need else None


def run(M, t, d, steps, coefficients, out=None):
    out = torch.full_like(d, 5.0) if out is None else out
    qa.qa_orthogonalize(M, code_of(t), d, steps, coefficients, out, room(M, t))
    return out


SHAPES = [(1, 1, 1, 0), (1, 1, 7, 0), (1, 9, 1, 2), (3, 5, 3, 0), (1, 32, 32, 0), (2, 33, 31, 1), (1, 64, 64, 8), (4, 65, 130, 0), (2, 130, 65, 3), (1, 200, 96, 0),
          (1, 96, 513, 0), (3, 127, 129, 0), (1, 300, 257, 7)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,R,C,pad", SHAPES)
@pytest.mark.parametrize("abc", [(1.0, 0.0, 0.0), (0.0, 1.0, 0.0), (0.0, 0.0, 1.0), (3.4445, -4.7750, 2.0315)])
def test_one_step(t, N, R, C, pad, abc):
    gen = gen_of(t, N, R, C, abc)
    v, d = matrices_of(gen, N, R, C, t, pad, lead=1, scale=1e-3)
    M = qa.Matrices.make(N, R, C, C + pad)
    out = run(M, t, d, 1, [abc])
    assert (out[:, :, C:] == 5.0).all()
    a, b, c = (abs(k) for k in abc)
    r = 2.0 ** -22                                                # of a number that is held
    for i in range(N):
        want = ref.orthogonal(v[i], 1, [abc])
        x = v[i] / torch.sqrt((v[i] * v[i]).sum())
        if R > C:
            x, want = x.t(), want.t()
        n, m = x.shape
        X = x.abs()
        s = lambda k: (3 * k / 16 + 16) * U + 2.0 ** -22 + 2 * r  # of a product's terms: sums, what is left out, both factors  # noqa: E731
        tiny = 2.0 ** -34
        A = X @ X.t()
        dA = s(m) * A + r * A + tiny * (1 + 2 * X.sum(dim=1, keepdim=True) + 2 * X.sum(dim=1))
        B = b * A + c * (A @ A)
        dB = b * dA + c * (2 * dA @ A + s(n) * A @ A) + r * B + tiny * (1 + 2 * c * (A.sum(dim=1, keepdim=True) + A.sum(dim=1)))
        tol = a * (r * X + tiny) + dB @ X + s(n) * (B @ X) + tiny * B.sum(dim=1, keepdim=True) + 2 * U * want.abs() + HALF_ULP[t] * 1.01 * want.abs()
        tol = tol + 2.0 ** -34 + (2.0 ** -24 if t == "f16" else 0.0)
        got = out[i, :, :C].cpu().to(F64)
        got = got.t() if R > C else got
        assert ((got - want).abs() <= tol).all(), (i, float(((got - want).abs() / tol).max()))


def off(got, want):
    return float((got - want).norm() / want.norm())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,R,C,pad", [(1, 1, 5, 0), (2, 40, 33, 0), (1, 128, 300, 4), (2, 500, 120, 0), (40, 72, 64, 0), (1, 700, 513, 1)])
def test_five_steps(t, N, R, C, pad):
    gen = gen_of("five", t, N, R, C)
    v, d = matrices_of(gen, N, R, C, t, pad, scale=30.0)
    out = run(qa.Matrices.make(N, R, C, C + pad), t, d, 5, None)
    for i in range(N):
        assert off(out[i, :, :C].cpu().to(F64), ref.orthogonal(v[i], 5)) <= 341 * 8 * U + HALF_ULP[t]


@pytest.mark.parametrize("t,N,R,C", [("f32", 1, 3500, 3300), ("bf16", 5, 1500, 1700)])
def test_large_tiles(t, N, R, C):
    """Enough tiles for those of 256 x 256, ends inside them; the reference on the device, where 64 bits are quick."""
    gen = gen_of("large", t)
    v, d = matrices_of(gen, N, R, C, t)
    out = run(qa.Matrices.make(N, R, C), t, d, 2, None)
    for i in {0, N - 1}:
        want = ref.orthogonal(v[i].to(DEV), 2)
        assert off(out[i].to(F64), want) <= 5 * 8 * U + HALF_ULP[t]
        rows = (out[i].to(F64) - want).norm(dim=1) / want.norm(dim=1)
        cols = (out[i].to(F64) - want).norm(dim=0) / want.norm(dim=0)
        assert float(rows.max()) < 5 * 32 * U + 2 * HALF_ULP[t] and float(cols.max()) < 5 * 32 * U + 2 * HALF_ULP[t]


def test_singular_values_come_near_one():
    gen = gen_of("svd")
    v, d = matrices_of(gen, 1, 200, 300, "f32")
    out = run(qa.Matrices.make(1, 200, 300), "f32", d, 5, None)
    s = torch.linalg.svdvals(out[0].cpu().to(F64))
    assert 0.5 < float(s.min()) and float(s.max()) < 1.3


def test_any_size_of_numbers_zeros_and_what_is_not_finite():
    gen = gen_of("sizes")
    v, d = matrices_of(gen, 6, 50, 70, "f32")
    M = qa.Matrices.make(6, 50, 70)
    plain = run(M, "f32", d, 3, None)
    e = d.clone()
    e[0] *= 2.0 ** 110
    e[1] *= 2.0 ** -100
    e[2] = 0.0
    e[3, 4, 5] = math.inf
    e[4, 49, 69] = math.nan
    got = run(M, "f32", e, 3, None)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1]) and torch.equal(got[5], plain[5])
    assert (got[2] == 0).all() and torch.isnan(got[3]).all() and torch.isnan(got[4]).all()


def test_in_place_and_a_schedule_of_coefficients():
    gen = gen_of("schedule")
    v, d = matrices_of(gen, 2, 60, 90, "f32")
    M = qa.Matrices.make(2, 60, 90)
    schedule = [(4.0, -6.0, 3.0), (3.0, -3.2, 1.2), (1.875, -1.25, 0.375)]
    away = run(M, "f32", d, 3, schedule)
    for i in range(2):
        assert off(away[i].cpu().to(F64), ref.orthogonal(v[i], 3, schedule)) <= 100 * 8 * U
    run(M, "f32", d, 3, schedule, out=d)
    assert torch.equal(d, away)


@pytest.mark.parametrize("N,R,C,pad", [(1, 40, 72, 0), (3, 97, 33, 5), (1, 300, 310, 0)])
@pytest.mark.parametrize("momentum,nesterov", [(True, 1), (True, 0), (False, 1)])
def test_step(N, R, C, pad, momentum, nesterov):
    gen = gen_of("step", N, R, C, momentum, nesterov)
    g, gd = matrices_of(gen, N, R, C, "f32", pad, 0, 1e-2)
    m, md = matrices_of(gen, N, R, C, "f32", pad, 0, 1e-2)
    x, xd = matrices_of(gen, N, R, C, "f32", pad, 0, 0.1)
    M = qa.Matrices.make(N, R, C, C + pad)
    ws = room(M, "f32")
    mu, eta, shrink = 0.95, 0.02, 0.99
    for _ in range(2):
        qa.qa_step_orthogonal(M, gd, md if momentum else None, xd, mu, nesterov, 5, None, eta, shrink, ws)
    assert (xd[:, :, C:] == 7.0).all() and (md[:, :, C:] == 7.0).all() and torch.equal(gd[:, :, :C].cpu().to(F64), g)
    f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    for i in range(N):
        wm, wx = m[i] if momentum else None, x[i]
        for _ in range(2):
            wm, wx = ref.step(g[i], wm, wx, f(mu), nesterov, 5, None, f(eta), f(shrink))
        if momentum:
            assert ((md[i, :, :C].cpu().to(F64) - wm).abs() <= 4 * U * (m[i].abs() + 2 * g[i].abs())).all()
        else:
            assert torch.equal(md[i, :, :C].cpu().to(F64), m[i])
        tol = 2 * eta * 341 * 8 * U * math.sqrt(min(R, C)) * 1.2
        assert float((xd[i, :, :C].cpu().to(F64) - wx).norm()) <= tol + 4 * U * float(x[i].norm())


def test_repeats_bit_for_bit():
    gen = gen_of("again")
    v, d = matrices_of(gen, 2, 333, 257, "f32")
    M = qa.Matrices.make(2, 333, 257)
    a = run(M, "f32", d, 5, None)
    assert torch.equal(a, run(M, "f32", d, 5, None))


def test_no_matrices():
    qa.qa_orthogonalize(qa.Matrices.make(0, 4, 4), qa.QA_F32, None, 5, None, None, None)


@pytest.mark.parametrize("N,R,C", [(2, 90, 70), (1, 300, 200)])
def test_captured_and_replayed_among_eager_steps(N, R, C):
    gen = gen_of("graph", R)
    g, gd = matrices_of(gen, N, R, C, "f32", 0, 0, 1e-2)
    _, x0 = matrices_of(gen, N, R, C, "f32", 0, 0, 0.1)
    M = qa.Matrices.make(N, R, C)
    ws = room(M, "f32")

    def step(g, m, x):
        qa.qa_step_orthogonal(M, g, m, x, 0.9, 1, 5, None, 0.02, 0.99, ws)
    m, x = torch.zeros_like(gd), x0.clone()
    want_m, want_x = torch.zeros_like(gd), x0.clone()
    other_m, other_x = torch.zeros_like(gd), x0.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(gd, other_m, other_x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(gd, m, x)
    for i in range(5):
        step(gd, want_m, want_x)
        step(-gd, other_m, other_x)                               # the same workspace, other numbers
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m, want_m) and torch.equal(x, want_x), i


def test_offsets_beyond_32_bits():
    """Rows 40000 elements apart, matrices 2^31 elements apart, at the end of the buffer."""
    gen = gen_of("far")
    R, C, stride, apart = 200, 150, 40000, (1 << 31) + 8
    v = torch.randn(2, R, C, generator=gen)
    flat = torch.empty(apart + R * stride, device=DEV)
    for i in range(2):
        flat[i * apart:i * apart + R * stride].view(R, stride)[:, :C] = v[i].to(DEV)
    M = qa.Matrices(2, R, C, stride, apart)
    run(M, "f32", flat, 3, None, out=flat)
    near = run(qa.Matrices.make(2, R, C), "f32", v.to(DEV), 3, None)
    for i in range(2):
        assert torch.equal(flat[i * apart:i * apart + R * stride].view(R, stride)[:, :C], near[i])


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("N,R,C", [(3, 128, 128), (2, 288, 96), (1, 64, 512), (1, 512, 64), (1, 129, 129), (1, 64, 513), (300, 17, 23)])
def test_sides_of_what_a_compute_unit_holds(t, N, R, C):
    gen = gen_of("held", t, N, R, C)
    v, d = matrices_of(gen, N, R, C, t)
    out = run(qa.Matrices.make(N, R, C), t, d, 5, None)
    for i in {0, N // 2, N - 1}:
        assert off(out[i].cpu().to(F64), ref.orthogonal(v[i], 5)) <= 341 * 8 * U + HALF_ULP[t]


def test_many_matrices_side_by_side():
    gen = gen_of("many")
    v, d = matrices_of(gen, 700, 40, 600, "bf16")
    out = run(qa.Matrices.make(700, 40, 600), "bf16", d, 5, None)
    for i in (0, 1, 350, 699):
        assert off(out[i].cpu().to(F64), ref.orthogonal(v[i], 5)) <= 341 * 8 * U + 2.0 ** -8
