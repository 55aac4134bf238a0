"""Gradient under an output layer where rows differ by many powers of two."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_output_layer import F64, TYPES, code_of, gen_of, inside, room

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
