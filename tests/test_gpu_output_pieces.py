"""Gradient under an output layer in pieces of the rows and of the vocabulary, with splits of dx's sums and rows that do not count in the same call.

Tolerances are those of test_gpu_output_layer.py; sums in 64 bits on the device, where they are quick."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_output_layer import F64, HALF_ULP, TYPES, U, code_of, dz_of, room

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")


def check(t, T, V, H, kept, entropy, accumulate):
    """kept: bool [T], the others' weights are 0 and their x is NaN."""
    gen = torch.Generator(device=DEV).manual_seed(T + V + H)
    w = (torch.randn(V, H, generator=gen, device=DEV) * (2 / math.sqrt(H))).to(TYPES[t])
    x = torch.randn(T, H, generator=gen, device=DEV).to(TYPES[t])
    y = torch.randint(0, V, (T,), generator=gen, device=DEV)
    a = -torch.rand(T, generator=gen, device=DEV) - 0.5
    e = 0.3 * torch.randn(T, generator=gen, device=DEV) if entropy else None
    kept = kept.to(DEV)
    a[~kept] = 0.0
    if entropy:
        e[~kept] = 0.0
    h, st = torch.zeros(T, device=DEV), torch.full((T, 2), math.nan, device=DEV)
    which = kept.nonzero()[:, 0]
    for rows in which.split(1000):
        _, _, hh, ss = ref.score(x[rows].to(F64), w.to(F64), y[rows])
        h[rows], st[rows] = hh.float(), ss.float()
    xd = x.clone()
    xd[~kept] = math.nan
    dx, dw = torch.full((T, H), 5.0, dtype=TYPES[t], device=DEV), torch.full((V, H), 3.0, device=DEV)
    layer = qa.OutputLayer.make(T, V, H)
    qa.qa_output_logprob_grad(layer, code_of(t), xd, w, y.to(torch.int32), st, h if entropy else None, a, e, dx, H, dw, H, int(accumulate),
                              room(layer, qa.QA_OP_LOGPROB_GRAD, t))
    assert (dx[~kept] == 0).all()
    w64, want_w = w.to(F64), torch.full((V, H), 3.0 if accumulate else 0.0, dtype=F64, device=DEV)
    off_w = torch.zeros_like(want_w)
    sums, part = (3 * max(T, V) / 16 + 64) * U, 2.0 ** -11 if t == "bf16" else 2.0 ** -21
    for rows in which.split(1000):
        x64, a64 = x[rows].to(F64), a[rows].to(F64)
        z, _, h64, st64 = ref.score(x64, w64, y[rows])
        c, _ = ref.logits_grad(z, y[rows], st[rows].to(F64), h[rows].to(F64), a64, e[rows].to(F64) if entropy else None)
        lp = z - st64[:, :1] - st64[:, 1:]
        off = dz_of(x64, w64, t)[:, None] + 8 * U * (z.abs() + st64[:, :1].abs() + st64[:, 1:]) + 2.0 ** -21
        size = a64.abs()[:, None] * torch.exp(lp) * off
        if entropy:
            size = size + e[rows].to(F64).abs()[:, None] * torch.exp(lp) * (lp.abs() + h64[:, None] + 1) * off
        size = size + 4 * U * c.abs()
        small = 2.0 ** -38 * (1.5 + (18 * float(e.abs().max()) if entropy else 0))
        want = c @ w64
        tol = (size + (part + 2.0 ** -21 + sums) * c.abs() + small) @ w64.abs() + 1.01 * HALF_ULP[t] * want.abs() + (2.0 ** -24 if t == "f16" else 0.0)
        assert ((dx[rows].to(F64) - want).abs() <= tol).all()
        want_w += c.t() @ x64
        # the parts of x: 2^-38 of the largest |g| |x| of a row, below 10 here
        off_w += (size + (2.0 ** -20 + sums) * c.abs() + small).t() @ x64.abs() + 10 * small * (c.abs() / a64.abs()[:, None]).sum(0)[:, None]
    assert ((dw.to(F64) - want_w).abs() <= off_w + 4 * U * want_w.abs()).all()


@pytest.mark.parametrize("t,T,V,H,entropy,accumulate", [("bf16", 66001, 1030, 40, True, False), ("f16", 131100, 1100, 32, False, True), ("f32", 70000, 1024, 20, False, False)])
def test_pieces_of_the_rows(t, T, V, H, entropy, accumulate):
    """More rows than one piece of c can have; dw goes on from piece to piece, and none of a piece's rows count or all do."""
    kept = torch.rand(T, generator=torch.Generator().manual_seed(1)) < 0.2
    kept[: T // 4] = True
    kept[T // 2 + 1000:] &= t != "f16"
    check(t, T, V, H, kept, entropy, accumulate)


@pytest.mark.parametrize("t,T,V,H", [("bf16", 20000, 20011, 32), ("bf16", 9000, 20011, 32), ("f16", 9000, 20011, 40), ("f32", 9000, 20011, 20)])
@pytest.mark.parametrize("some", [0.0002, 0.07, 0.5])
def test_pieces_of_the_vocabulary_where_some_rows_count(t, T, V, H, some):
    """Several pieces, the last one shorter, and dx's sums in splits, whose number the device finds for the rows that count."""
    kept = torch.rand(T, generator=torch.Generator().manual_seed(2)) < some
    kept[T - 1] = True
    check(t, T, V, H, kept, False, False)
