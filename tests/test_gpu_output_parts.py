"""What two binary16 parts and powers of two as scales keep, under an output layer (tolerances: test_gpu_output_scales.py)."""
import math

import pytest
import torch

from test_gpu_output_layer import TYPES, check_score, code_of, gen_of, inside, layer_of, room, score
from test_gpu_output_scales import check, rows_of

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")


@pytest.mark.parametrize("t,lead", [("f32", 0), ("f16", 0), ("f16", 1), ("bf16", 0)])
def test_words_that_are_nearly_alike(t, lead):
    """w = 1 + small: c sums to 0 in each row, so that dx is some 2^-6 of its terms, and a rounding of c by 2^-12 (one part) would be a quarter of a
    percent of it; binary16 has 2^-11.  Small x, as the logits' own roundings count too."""
    gen = gen_of("alike", t)
    T, V, H = 100, 300, 64
    x, w, y = rows_of(gen, T, V, H)
    check(t, x * 2.0 ** -8, 1 + w * 2.0 ** -5, y, torch.rand(T, generator=gen) + 0.5, None, lead)


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 60])
def test_scoring_of_any_size(scale):
    """x small by as much as w is large: the same logits to the bit, in rows that are scaled too (more than 64)."""
    gen = gen_of("sizes")
    layer, x, xd, w, wd, y = layer_of(gen, 100, 200, 50, "f32")
    a, b = score(layer, xd, wd, y, "f32"), score(layer, xd * scale, wd / scale, y, "f32")
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_scoring_of_rows_of_many_sizes():
    gen = gen_of("row sizes")
    T, V, H = 130, 700, 100
    x, w, y = rows_of(gen, T, V, H)
    x *= 2.0 ** -torch.randint(0, 60, (T, 1), generator=gen).float()
    w *= 2.0 ** -torch.randint(0, 60, (V, 1), generator=gen).float()
    x64, xd = inside(x, "f32")
    w64, wd = inside(w, "f32")
    check_score("f32", x64, w64, y, score(qa.OutputLayer.make(T, V, H), xd, wd, y, "f32"))


@pytest.mark.parametrize("t,lead,T", [("f32", 0, 100), ("f32", 0, 40), ("bf16", 1, 100)])
@pytest.mark.parametrize("power", [-60, 60])
def test_gradient_of_any_size(t, lead, T, power):
    """x by s and w by 1 / s: the same c, dx by 1 / s and dw by s, to the bit; and both by g's own power."""
    gen = gen_of("gradient sizes", t, T)
    V, H = 300, 50
    layer, _, xd, _, wd, y = layer_of(gen, T, V, H, t, 0, lead)
    a = torch.rand(T, generator=gen).to(DEV)
    y = y.to(torch.int32).to(DEV)
    h, st = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
    qa.qa_output_logprob(layer, code_of(t), xd, wd, None, None, h, st, room(layer, qa.QA_OP_LOGPROB, t))
    got = []
    for s, g in ((1.0, 1.0), (2.0 ** power, 1.0), (1.0, 2.0 ** (power // 2))):
        x, w = torch.empty(T * H + 8, dtype=TYPES[t], device=DEV)[lead:lead + T * H].view(T, H), torch.empty(V * H + 8, dtype=TYPES[t], device=DEV)[lead:lead + V * H].view(V, H)
        x.copy_(xd * s), w.copy_(wd / s)
        dx, dw = torch.empty(T, H, dtype=TYPES[t], device=DEV), torch.empty(V, H, device=DEV)
        qa.qa_output_logprob_grad(layer, code_of(t), x, w, y, st, h, a * g, a * g, dx, H, dw, H, 0, room(layer, qa.QA_OP_LOGPROB_GRAD, t))
        got.append((dx * (s / g), dw / (s * g)))
    assert all(bool(torch.isfinite(v).all()) for v in got[0]) and float(got[0][1].abs().max()) > 0.01
    for other in got[1:]:
        assert torch.equal(other[0], got[0][0]) and torch.equal(other[1], got[0][1])
