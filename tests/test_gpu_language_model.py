"""The operators together, as the example runs them: the whole model's gradient against differences, and a short training."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decentral_lm", os.path.join(ROOT, "examples", "decentral_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradient_of_the_whole_model_by_differences():
    # directional central differences: the loss is good to about 2e-6 (fp32, means over 60 words), its slope along a unit
    # direction times the step 0.02 is some 1e-2, the third-order term below 1e-3 of it
    M = example()
    model = M.Model(40, 16)
    gen = torch.Generator(device="cuda").manual_seed(3)
    X = torch.empty((2, model.ld), device="cuda").normal_(0.0, 0.2, generator=gen)
    G = torch.zeros_like(X)
    text = torch.randint(0, 40, (2, 5, 13), generator=gen, device="cuda")
    model.gradient(X, G, text[..., :-1], text[..., 1:])
    for name, view in model.views(G).items():
        assert float(view.abs().max()) > 0, name
        direction = torch.zeros_like(X)
        model.views(direction)[name].copy_(view / view.flatten(1).norm(dim=1).view(-1, *[1] * (view.dim() - 1)))
        h = 0.02
        up, down = (model.gradient(X + s * h * direction, torch.zeros_like(G), text[..., :-1], text[..., 1:]) for s in (1, -1))
        slope = (up - down) / (2 * h)
        want = (G * direction).sum(1)
        assert bool(((slope - want).abs() <= 0.02 * want.abs() + 4e-4).all()), (name, slope, want)


def test_a_short_training_learns_the_chain():
    begin, end, consensus, allowed = example().run(steps=120, log=lambda *a: None)
    assert all(abs(v - math.log(500)) < 1.0 for v in begin)        # guessing
    assert max(end) < 0.5 * min(begin) and math.isfinite(consensus)
    assert allowed > 0.8
