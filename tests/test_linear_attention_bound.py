"""What the tolerance of linear attention's results in fp32 tells apart, without a GPU."""
import pytest
import torch

from tests.linear_attention import NAMES, squares, tolerance
from tests.test_gpu_linear_attention import reference


@pytest.mark.parametrize("N, dk, dv", [(1, 32, 48), (8, 64, 64), (40, 50, 50), (150, 16, 24)])
def test_operands_of_17_bits_are_beyond_the_tolerance(N, dk, dv):
    gen = torch.Generator().manual_seed(N)
    rand = lambda *shape: torch.empty(shape, dtype=torch.float32).normal_(0.0, 1.0, generator=gen)  # noqa: E731
    q, k, dy = rand(2, N, 2, dk), rand(2, N, 2, dk), rand(2, N, 2, dv)
    v, h0, dlast = rand(2, N, 2, dv), rand(2, 2, dk, dv), rand(2, 2, dk, dv)
    g, n = -torch.rand((2, N, 2), generator=gen) * 0.5, torch.full((2,), N)
    args = (q, k, v, g, h0, n, dy, dlast)
    exact, sizes, allowed = reference(*args), squares(reference, *args), tolerance(dk, dv, N)

    def bits(x, count):      # rounded to so many
        m, e = torch.frexp(x.double())
        return torch.ldexp(torch.round(m * 2.0 ** count), e - count)

    for count, beyond in ((17, True), (23, False)):
        off = reference(*(bits(x, count) for x in (q, k, v)), g, bits(h0, count), n, bits(dy, count), bits(dlast, count))
        for name in NAMES:
            error = float((off[name] - exact[name]).norm()) / float(sizes[name].norm())
            assert (error > allowed) == beyond, (name, count, error, allowed)
