"""The output layer's operators and the orthogonal step as the example's model uses them: with the norm in front of them, the 2-bit
messages behind them, and the parameters that they step."""
import importlib.util
import math
import os

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("next_token", os.path.join(ROOT, "examples", "next_token.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradient_without_kept_logits(example):
    """The same gradient as with them: logits, and their gradient, were rounded to bfloat16 there (2^-8 each, some 1/100 of a gradient together)."""
    got = {}
    for keep in (True, False):
        model = example.Model(131, 96, 2, 500, keep_logits=keep)
        x = model.initial(3)
        gen = torch.Generator(device=DEV).manual_seed(4)
        before = torch.randint(0, 131, (500,), generator=gen, device=DEV)
        after = torch.randint(0, 131, (500,), generator=gen, device=DEV).to(torch.int32)
        g = torch.full_like(x, math.nan)
        model.gradient(x, g, before, after)
        got[keep] = {n: model.view(g, n).double().cpu() for n in model.shape}, model.logprob.double().cpu(), model.entropy.double().cpu()
    for n in got[True][0]:
        a, b = got[True][0][n], got[False][0][n]
        assert bool(torch.isfinite(b).all()) and float((a - b).norm() / a.norm()) < 0.03, n
    assert float((got[True][1] - got[False][1]).abs().max()) < 0.05 and float((got[True][2] - got[False][2]).abs().max()) < 0.05


def test_matrix_steps_from_messages(example):
    """The average of a matrix's messages is read where it lies among the others', and nothing but the matrix is stepped."""
    workers, width = 3, 80
    model = example.Model(61, width, 2, 64, keep_logits=False)
    gen = torch.Generator(device=DEV).manual_seed(5)
    g = 1e-2 * torch.randn(workers, model.d, generator=gen, device=DEV)
    table = torch.empty(qa.qa_segment_plan_bytes(model.d, len(model.begin)), dtype=torch.uint8, device=DEV)
    plan = qa.qa_segment_plan_init(model.d, model.begin, model.length, table)
    L = qa.Layout.make(model.d, workers, 0, scale_stride=len(model.begin))
    codes, scales = torch.empty(workers, L.code_stride, dtype=torch.int32, device=DEV), torch.empty(workers, L.scale_stride, device=DEV)
    ws = torch.empty(max(256, qa.qa_segment_workspace_bytes(plan, workers, qa.QA_OP_QUANTIZE)), dtype=torch.uint8, device=DEV)
    qa.qa_quantize_pack_segments(L, plan, g, model.d, codes, scales, None, ws)
    x = model.initial(1)
    was = x.clone()
    example.MatrixSteps(model, ["w0", "w1"], workers, L).step(codes, scales, x, 0.02)
    fields = torch.stack([codes >> (2 * i) & 3 for i in range(16)], dim=-1).view(workers, -1)[:, :model.d].cpu().double()
    sign = torch.where(fields == 1, 1.0, torch.where(fields == 3, -1.0, 0.0))
    for i, n in enumerate(model.shape):
        at, shape = model.shape[n]
        end = at + math.prod(shape)
        if n not in ("w0", "w1"):
            assert torch.equal(x[at:end], was[at:end]), n
            continue
        mean = (sign[:, at:end] * scales[:, i].cpu().double()[:, None]).mean(dim=0).view(shape)
        _, want = ref.step(mean, torch.zeros_like(mean), was[at:end].view(shape).cpu().double(), 0.9, 1, 5, None, 0.02, 1.0)
        assert float((x[at:end].view(shape).cpu().double() - want).norm() / (want - was[at:end].view(shape).cpu().double()).norm()) < 1e-3


@pytest.mark.parametrize("keep_logits,orthogonal", [(False, False), (False, True), (True, True)])
def test_training_runs(example, keep_logits, orthogonal):
    losses, least = example.train(steps=8, workers=2, rows=256, vocab=67, width=64, layers=2, say=None, keep_logits=keep_logits, orthogonal=orthogonal)
    assert len(losses) == 8 and all(math.isfinite(v) for v in losses) and least > 0
