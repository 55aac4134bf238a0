"""Gradient under an output layer where rows differ by many powers of two: in x, in w, and in what they weigh.

Tolerances are those of test_gpu_output_layer.py, row by row.  With u = 2^-24 and everything per row t of x or v of w:
    z      off by dz = ((P K / 16 + 16) u + (P == 3) 2^-21) sum|x_t w_v|, and by what binary16 has no bits for in a row that is scaled by its
           largest magnitude: 2^-38 (max|x_t| sum|w_v| + max|w_v| sum|x_t|)
    c      off by p (dz + 8 u (|z| + |m| + log sum) + 2^-21) |g_t|, but never by more than 2 |g_t|; 2^-21 of it and 2^-38 |g_t| as two binary16 parts,
           2^-11 of it as one (dx of bfloat16)
    dx     the parts of w: 2^-21 of each, and 2^-38 of the largest |w|
    dw     the parts of x: 2^-21 of each, and 2^-38 of the largest |g_t| max|x_t| of all rows, times |c_tv| / |g_t|."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_output_layer import F64, HALF_ULP, TYPES, U, code_of, gen_of, inside, room

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")


def rows_of(gen, T, V, H):
    w = torch.randn(V, H, generator=gen) * (2 / math.sqrt(H))
    return torch.randn(T, H, generator=gen), w, torch.randint(0, V, (T,), generator=gen)


def gradient(t, x, w, y, st, h, a, e, lead):
    """-> x and w as they were rounded, dx and dw; rows that begin on no 16 bytes where lead is odd."""
    T, V, H = x.shape[0], w.shape[0], x.shape[1]
    x64, xd = inside(x, t, 0, lead)
    w64, wd = inside(w, t, 0, lead)
    if st is None:
        _, _, h64, st64 = ref.score(x64, w64, y)
        st, h = st64.float(), h64.float()
    layer = qa.OutputLayer.make(T, V, H)
    dx, dw = torch.full((T, H), 5.0, dtype=TYPES[t], device=DEV), torch.full((V, H), 5.0, device=DEV)
    qa.qa_output_logprob_grad(layer, code_of(t), xd, wd, y.to(torch.int32).to(DEV), st.to(DEV), h.to(DEV) if e is not None else None, a.to(DEV),
                              e.to(DEV) if e is not None else None, dx, H, dw, H, 0, room(layer, qa.QA_OP_LOGPROB_GRAD, t))
    return x64, w64, st, h, dx.cpu().to(F64), dw.cpu().to(F64)


def check(t, x, w, y, a, e=None, lead=0, dx_rows=slice(None)):
    x, w, _, _, got_dx, got_dw = gradient(t, x, w, y, None, None, a, e, lead)
    z, _, h, st = ref.score(x, w, y)
    a, e = a.to(F64), None if e is None else e.to(F64)
    c, _ = ref.logits_grad(z, y, st, h, a, e)                     # of exact statistics: a large row's are off by more than 1 in binary32
    T, V, H, P = x.shape[0], w.shape[0], x.shape[1], 3 if t == "f32" else 1
    X, W = x.abs(), w.abs()
    dz = ((P * H / 16 + 16) * U + (2.0 ** -21 if P == 3 else 0.0)) * (X @ W.t())
    dz = dz + 2.0 ** -38 * (X.amax(1)[:, None] * W.sum(1)[None] + X.sum(1)[:, None] * W.amax(1)[None])
    off = dz + 8 * U * (z.abs() + st[:, :1].abs() + st[:, 1:]) + 2.0 ** -21
    lp = z - st[:, :1] - st[:, 1:]
    p = torch.exp(lp + torch.clamp(off, max=50.0)).clamp(max=1.0)                   # as large as it can come out
    most = a.abs() + (18 * e.abs() if e is not None else 0)
    size = a.abs()[:, None] * p * off
    if e is not None:
        size = size + e.abs()[:, None] * p * (lp.abs() + h[:, None] + 1) * off
    size = torch.minimum(size, 2 * most[:, None]) + 4 * U * c.abs()
    sums = (3 * max(T, V) / 16 + 64) * U
    small = 2.0 ** -38 * most[:, None]
    part = 2.0 ** -11 if t == "bf16" else 2.0 ** -21
    want = c @ w
    tol = (size + (part + 2.0 ** -21 + sums) * c.abs() + small) @ W + 2.0 ** -38 * W.max() * c.abs().sum(1)[:, None] + HALF_ULP[t] * 1.01 * want.abs()
    tol = tol + (2.0 ** -24 if t == "f16" else 0.0)
    worst = ((got_dx - want).abs() / tol)[dx_rows]
    assert (worst <= 1).all(), ("dx", float(worst.max()), worst.amax(1).tolist()[:20])
    want = c.t() @ x
    lost = 2.0 ** -38 * float((most * X.amax(1)).max()) * (c.abs() / most.clamp(min=1e-300)[:, None]).sum(0)
    tol = (size + (2.0 ** -20 + sums) * c.abs() + small).t() @ X + lost[:, None] + 2 * U * want.abs()
    worst = (got_dw - want).abs() / tol
    assert (worst <= 1).all(), ("dw", float(worst.max()))


@pytest.mark.parametrize("t,lead", [("f32", 0), ("bf16", 0), ("bf16", 1), ("f16", 0), ("f16", 1)])
def test_logits_that_statistics_know_to_a_few_units_only(t, lead):
    """Logits of 10^8 (binary16: 10^4): a row's statistics and its logits, multiplied again, are some units apart, and exp of their difference is no
    probability.  No more than 1 comes of it, and nothing that is not finite, for the row or for dw."""
    gen = gen_of("far logits", t)
    T, V, H = 100, 300, 64
    x, w, y = rows_of(gen, T, V, H)
    x[::5] *= 2.0 ** (24 if t != "f16" else 10)
    a = torch.rand(T, generator=gen) + 0.5
    x64, _ = inside(x, t)
    w64, _ = inside(w, t)
    _, _, h, st = ref.score(x64, w64, y)
    st = st.float()
    st[::5, 0] -= 2.0 ** -22 * st[::5, 0].abs()                   # two units of binary32
    _, _, _, _, dx, dw = gradient(t, x, w, y, st, h.float(), a, None, lead)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    # |c| <= |a| in each number, and no row's c sum to more than two of it but for those close to the largest
    near = (x64 @ w64.t() >= st.to(F64)[:, :1] - 200).sum(1) + 1
    assert (dx.abs() <= 1.01 * (a[:, None] * near[:, None] * w64.abs().max()).to(F64)).all()


@pytest.mark.parametrize("t,lead,T", [("f32", 0, 100), ("f32", 0, 40), ("bf16", 0, 100), ("bf16", 1, 100), ("f16", 0, 100), ("f16", 1, 40)])
@pytest.mark.parametrize("entropy", [False, True])
def test_rows_that_weigh_little_beside_others(t, lead, T, entropy):
    """Weights from 1 to 2^-40: each row's dx is as exact as if it were alone."""
    gen = gen_of("weights", t, T, entropy)
    x, w, y = rows_of(gen, T, 300, 96)
    weight = 2.0 ** -torch.randint(0, 41 if t != "f16" else 13, (T,), generator=gen).float()
    a = -(torch.rand(T, generator=gen) + 0.5) * weight * (64 if t == "f16" else 1)
    check(t, x, w, y, a, 0.3 * torch.randn(T, generator=gen) * weight if entropy else None, lead)


@pytest.mark.parametrize("t,lead,T", [("f32", 0, 100), ("f32", 0, 40), ("bf16", 0, 100), ("bf16", 1, 100), ("f16", 1, 100)])
def test_a_row_of_x_beside_a_much_larger_one(t, lead, T):
    """One row 2^34 times as large as the others (binary16: 2^8), and one as small: the others' logits are as exact as without it."""
    gen = gen_of("large row", t, T)
    x, w, y = rows_of(gen, T, 300, 96)
    x[T // 2] *= 2.0 ** (34 if t != "f16" else 8)
    x[3] *= 2.0 ** (-34 if t != "f16" else -8)
    check(t, x, w, y, torch.rand(T, generator=gen) + 0.5, None, lead)


@pytest.mark.parametrize("t,lead,T", [("f32", 0, 100), ("f32", 0, 40), ("bf16", 0, 100), ("bf16", 1, 100), ("f16", 1, 100)])
@pytest.mark.parametrize("power", [10, 30, 60])
def test_a_row_of_w_beside_a_much_larger_one(t, lead, T, power):
    """A word whose logits are 2^30 below all others', and one with a small row: the others' logits, and dw, are as exact as without them."""
    gen = gen_of("large word", t, T, power)
    x, w, y = rows_of(gen, T, 300, 96)
    power = power if t != "f16" else power // 4
    x[:, 0] = 1.0
    w[150] *= 2.0 ** -20 if t != "f16" else 2.0 ** -8
    w[150, 0] = -(2.0 ** power)
    w[7] *= 2.0 ** -30 if t != "f16" else 2.0 ** -8
    y[y == 150] = 3
    check(t, x, w, y, torch.rand(T, generator=gen) + 0.5, None, lead)


@pytest.mark.parametrize("t,lead", [("f32", 0), ("bf16", 1)])
def test_replayed_where_logits_become_large(t, lead):
    """A captured gradient whose logits are small, then large, then small: each replay is what an eager call gives, bit for bit."""
    gen = gen_of("replayed scales", t)
    T, V, H = 100, 3000, 64
    x, w, y = rows_of(gen, T, V, H)
    _, xd = inside(x, t, 0, lead)
    _, wd = inside(w, t, 0, lead)
    y, a = y.to(torch.int32).to(DEV), torch.rand(T, generator=gen).to(DEV)
    layer = qa.OutputLayer.make(T, V, H)
    h, st = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
    ws, ws2 = room(layer, qa.QA_OP_LOGPROB, t), room(layer, qa.QA_OP_LOGPROB_GRAD, t)
    dx, dw = torch.empty(T, H, dtype=TYPES[t], device=DEV), torch.empty(V, H, device=DEV)

    def both():
        qa.qa_output_logprob(layer, code_of(t), xd, wd, None, None, h, st, ws)
        qa.qa_output_logprob_grad(layer, code_of(t), xd, wd, y, st, h, a, a, dx, H, dw, H, 0, ws2)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for power in (0, 20, 0, 30, 40, 0):
        xd[::7] *= 2.0 ** power
        both()
        torch.cuda.synchronize()
        want = dx.clone(), dw.clone()
        dx.fill_(7.0), dw.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and bool(torch.isfinite(dw).all()), power
        xd[::7] *= 2.0 ** -power


@pytest.mark.parametrize("t,lead", [("f32", 0), ("bf16", 1), ("bf16", 0), ("f16", 0), ("f16", 1)])
@pytest.mark.parametrize("power", [0, 30])
def test_one_side_is_as_both(t, lead, power):
    """dx alone and dw alone, of small logits and large ones, are what both together are, bit for bit."""
    gen = gen_of("one side", t)
    T, V, H = 150, 500, 64
    x, w, y = rows_of(gen, T, V, H)
    w[7] *= 2.0 ** (power if t != "f16" else power // 4)
    x64, xd = inside(x, t, 0, lead)
    w64, wd = inside(w, t, 0, lead)
    _, _, h, st = (v.float().to(DEV) if v.dim() <= 2 else v for v in ref.score(x64, w64, y))
    y, a = y.to(torch.int32).to(DEV), torch.rand(T, generator=gen).to(DEV)
    layer = qa.OutputLayer.make(T, V, H)
    got = []
    for wants in ("xw", "x", "w"):
        dx = torch.full((T, H), 5.0, dtype=TYPES[t], device=DEV) if "x" in wants else None
        dw = torch.full((V, H), 5.0, device=DEV) if "w" in wants else None
        qa.qa_output_logprob_grad(layer, code_of(t), xd, wd, y, st, h, a, a, dx, H, dw, H, 0, room(layer, qa.QA_OP_LOGPROB_GRAD, t))
        got.append((dx, dw))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[2][1])
