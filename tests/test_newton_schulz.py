"""The bounds that the GPU tests of orthogonalised matrices use, and what the header promises of them, without a GPU."""
import os
import re

import pytest
import torch

from tests.newton_schulz import A, B, C, MOST, SLOPE, iterate, matrices, tolerance

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("shape", [(16, 16), (17, 33), (63, 64), (130, 70), (200, 333), (50, 2000), (2000, 50), (513, 640), (700, 650), (256, 256)])
def test_operands_of_one_number_of_16_bits_are_beyond_the_tolerance(shape):
    x = matrices((1, *shape), seed=sum(shape), device="cpu")

    def one(v):
        return (v * 8192).half().double() / 8192

    def two(v):
        high = (v * 8192).half().double()
        return (high + (v * 8192 - high).half().double()) / 8192

    for iterations in (1, 2):
        exact = iterate(x, iterations)
        allowed = tolerance(exact, iterations)
        assert float((iterate(x, iterations, one) - exact).norm()) > 3 * allowed
        assert float((iterate(x, iterations, two) - exact).norm()) < 0.1 * allowed
    exact = iterate(x, 5)
    assert tolerance(exact, 5) < 0.01 * float(exact.norm())


def test_constants_of_the_tolerance():
    x = torch.linspace(0.0, MOST, 1_000_001, dtype=torch.float64)
    f, slope = A * x + B * x ** 3 + C * x ** 5, A + 3 * B * x ** 2 + 5 * C * x ** 4
    assert float(f.min()) >= 0 and float(f.max()) <= MOST
    assert float(slope.abs().max()) <= SLOPE and float((f[1:] / x[1:]).max()) <= 3.45
    assert float((B * x + C * x ** 3).abs().max()) * MOST <= 9.4


def test_singular_values_end_in_the_stated_range():
    # what the header and the docstring say
    for path in ("include/choco_train.h", "paper_1907_09356_amd/train.py"):
        text = re.sub(r"\s+\**\s*", " ", open(os.path.join(ROOT, path)).read())
        low, high, part = re.search(r"(0\.\d+) \.\. (1\.\d+) after five[^.]*?1 / (\d+) of", text).groups()
        x = torch.logspace(-torch.log10(torch.tensor(float(part))).item(), 0, 1_000_001, dtype=torch.float64)
        for _ in range(5):
            x = A * x + B * x ** 3 + C * x ** 5
        assert float(low) <= float(x.min()) <= float(low) + 0.01 and float(high) - 0.01 <= float(x.max()) <= float(high), path
