"""Linear attention and the orthogonalising optimiser together, as the example runs them beside the lookups, AdamW and gossip: the whole
model's gradient against differences, and a run of every combination."""
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
    model = M.Model(40, 16, "attention", heads=2)
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


@pytest.mark.parametrize("mixer, optimiser", [("attention", "adamw"), ("attention", "muon"), ("recurrence", "muon")])
def test_runs(mixer, optimiser):
    begin, end, consensus, allowed = example().run(steps=8, workers=3, log=lambda *a: None, mixer=mixer, optimiser=optimiser)
    assert all(math.isfinite(v) for v in begin + end + [consensus, allowed]) and 0.0 <= allowed <= 1.0


def test_token_by_token_continues_what_the_prompt_left():
    # the same words at once: a token's output follows from the state that the ones before it left
    M = example()
    model = M.Model(50, 32, "attention")
    gen = torch.Generator(device="cuda").manual_seed(5)
    X = torch.empty((1, model.ld), device="cuda").normal_(0.0, 0.2, generator=gen)
    prompt = torch.randint(0, 50, (3, 9), generator=gen, device="cuda")
    words = model.generate(X, prompt, 6)
    y = model.forward(X, torch.cat((prompt, words), 1)[None])[0].view(3, 15, 32)
    p = model.views(X)
    logits = y[:, 8:14] @ p["table"][0].t() + p["bias"][0]
    best = logits.gather(2, words[..., None])[..., 0]
    # sums of some hundred products in another order
    assert bool((best >= logits.amax(2) - 1e-3 * logits.abs().amax()).all())
