"""The operators together: the example's language model, its gradient against automatic differentiation in 64 bits, and its training."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("next_token", os.path.join(ROOT, "examples", "next_token.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def loss_in_64_bits(model, x, before, after):
    at = lambda n: model.view(x, n)  # noqa: E731

    def norm(h, w):
        return h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * w
    h = at("embedding")[before]
    for i in range(model.layers):
        h = h + norm(h, at(f"norm{i}")) @ at(f"w{i}").t()
    logits = norm(h, at("norm_out")) @ at("w_out").t()
    return -torch.log_softmax(logits, dim=1).gather(1, after.long()[:, None]).mean()


def test_gradient_of_the_whole_model(example):
    """Each activation is rounded to 8 bits of a magnitude or to bfloat16, by 1/126 and 1/256 at most: independent errors of less than a
    hundredth per factor, of which a gradient has some five."""
    model = example.Model(61, 80, 2, 700)
    x = model.initial(3)
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    before = torch.randint(0, 61, (700,), generator=gen, device="cuda:0")
    after = torch.randint(0, 61, (700,), generator=gen, device="cuda:0").to(torch.int32)
    g = torch.full_like(x, math.nan)
    model.gradient(x, g, before, after)
    x64 = x.double().cpu().requires_grad_(True)
    loss = loss_in_64_bits(model, x64, before.cpu(), after.cpu())
    loss.backward()
    assert abs(float(-model.logprob.mean()) - float(loss.detach())) < 0.02
    for name in model.shape:
        want, got = model.view(x64.grad, name), model.view(g, name).double().cpu()
        assert float((got - want).norm() / want.norm()) < 0.03, name


def test_training_with_two_bit_messages(example):
    losses, least = example.train(steps=120, workers=2, rows=1024, vocab=129, width=64, layers=2, eta=0.02, say=None)
    assert abs(losses[0] - math.log(129)) < 1.0
    assert sum(losses[-10:]) / 10 < least + 0.35 * (losses[0] - least)
