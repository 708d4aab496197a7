"""Orthogonalised matrices and steps along them against the iteration in 64 bits, to what operands as two fp16 numbers allow (`tolerance`; one number for
an operand is far beyond it), with tiles of every size."""
import math

import numpy as np
import pytest
import torch

from paper_1907_09356_amd import train as T
from tests.newton_schulz import MOST, SLOPE, iterate, matrices, tolerance

pytestmark = pytest.mark.gpu

# (batch, rows, cols): taken whole by a workgroup; in tiles of 64; of 128; and X' in tiles of 128, P and Q of 64
WHOLE = [(3, 1, 1), (2, 7, 5), (3, 16, 16), (2, 17, 33), (3, 64, 63), (2, 64, 192), (2, 192, 64), (2, 64, 100), (2, 32, 512), (1, 1, 500)]
SIXTY_FOUR = [(2, 128, 128), (1, 130, 70), (1, 333, 1000), (1, 1000, 333), (3, 200, 333), (2, 513, 640), (2, 50, 2000), (2, 2000, 50), (1, 1, 600), (1, 700, 129)]
LARGE = [(20, 700, 650), (20, 650, 700), (64, 256, 256), (70, 260, 200), (10, 1024, 640), (10, 640, 1024), (60, 129, 700), (60, 700, 129)]
BOTH = [(2, 650, 2600), (2, 2600, 650), (1, 700, 5000), (1, 5000, 700)]


@pytest.mark.parametrize("shape", WHOLE + SIXTY_FOUR + LARGE + BOTH)
@pytest.mark.parametrize("iterations", [1, 2, 5])
def test_as_near_as_two_numbers_of_16_bits_allow(shape, iterations):
    x = matrices(shape, seed=sum(shape))
    got = T.orthogonalize(x, iterations=iterations).double()
    for part in range(0, shape[0], 10):
        exact = iterate(x[part:part + 10], iterations)
        off = float((got[part:part + 10] - exact).flatten(1).norm(dim=1).max())
        assert off <= tolerance(exact, iterations), (part, off, tolerance(exact, iterations))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(2, 60, 90), (2, 333, 200), (20, 700, 650), (20, 650, 700)])
def test_inputs_of_16_bits(dtype, shape):
    x = matrices(shape, dtype=dtype)
    for iterations in (1, 2):
        exact = iterate(x, iterations)
        assert float((T.orthogonalize(x, iterations=iterations).double() - exact).flatten(1).norm(dim=1).max()) <= tolerance(exact, iterations)


@pytest.mark.parametrize("n, shapes, grad", [
    (20, [(700, 650), (650, 700)], torch.float32), (20, [(700, 650), (650, 700)], torch.bfloat16), (2, [(2600, 650), (650, 1300)], torch.float32),
    (3, [(64, 192), (130, 70), (192, 64)], torch.bfloat16), (1, [(333, 1000)], torch.float32),
])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("iterations", [1, 2])
def test_steps_as_near_as_two_numbers_of_16_bits_allow(n, shapes, grad, nesterov, iterations):
    start, at = [], 5
    for r, c in shapes:
        start.append(at)
        at += r * c + 3
    ld = (at + 63) // 64 * 64
    gen = torch.Generator(device="cuda").manual_seed(n)
    X = torch.empty((n, ld), device="cuda").normal_(0.0, 0.05, generator=gen)
    clip = torch.rand(n, device="cuda", generator=gen) + 0.5
    opt = T.Muon(X, at, (np.array(start), [s[0] for s in shapes], [s[1] for s in shapes]), momentum=0.9, nesterov=nesterov, weight_decay=0.1, iterations=iterations)
    moments = [0.0 for _ in shapes]
    for _ in range(2):
        before = X.double()
        G = torch.zeros((n, ld), device="cuda", dtype=grad)
        for i, (a, (r, c)) in enumerate(zip(start, shapes)):
            G[:, a:a + r * c] = matrices((n, r, c), seed=i + n).flatten(1).to(grad)
        opt.step(G, 0.5, grad_scale=clip)
        for i, (a, (r, c)) in enumerate(zip(start, shapes)):
            g = G[:, a:a + r * c].double().view(n, r, c) * clip.double()[:, None, None]
            moments[i] = 0.9 * moments[i] + g
            exact = iterate(g + 0.9 * moments[i] if nesterov else moments[i], iterations)
            rate = 0.5 * math.sqrt(max(1.0, r / c))
            want = before[:, a:a + r * c].view(n, r, c) * (1 - 0.5 * 0.1) - rate * exact
            off = float((X[:, a:a + r * c].double().view(n, r, c) - want).flatten(1).norm(dim=1).max())
            # momentum and what is orthogonalised: five roundings more of the first X, each 2^-24, of at most four times it (g + 0.9 m: of terms as long as
            # 1.9 + 0.9^2 times g); x: three roundings
            allowed = rate * tolerance(exact, iterations, begin=2.0 ** -22 + 20 * 2.0 ** -24) + 3 * 2.0 ** -24 * float(want.flatten(1).norm(dim=1).max())
            assert off <= allowed, (r, c, off, allowed)


def test_rounds_of_many_workers_against_64_bits():
    # operands of 230 workers are more than a round's
    n, r, c = 230, 700, 800
    G = torch.empty((n, r * c), device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    X = torch.zeros((n, r * c), device="cuda")
    T.Muon(X, r * c, ([0], [r], [c]), momentum=0.0, nesterov=False, iterations=2).step(G, 1.0)
    stack = T.orthogonalize(G.view(n, r, c), iterations=2)
    for w in (0, 1, 63, 64, 114, 115, 116, n - 1):
        exact = iterate(G[w].view(1, r, c), 2)[0]
        allowed = tolerance(exact[None], 2)
        assert float((-X[w].double().view(r, c) - exact).norm()) <= allowed and float((stack[w].double() - exact).norm()) <= allowed


def test_singular_values_lie_in_the_stated_range():
    # from 1/500 of the norm on between 0.68 and 1.21, five iterations' error aside
    gen = torch.Generator(device="cuda").manual_seed(5)
    q1 = torch.linalg.qr(torch.randn(150, 150, device="cuda", dtype=torch.float64, generator=gen))[0]
    q2 = torch.linalg.qr(torch.randn(260, 260, device="cuda", dtype=torch.float64, generator=gen))[0][:150]
    for first, rest in ((1.0, 0.05), (1.0, 0.002), (0.7, 0.7), (0.3, 0.3)):      # one value, and others from 1/400 of the norm to so much of it
        s = torch.cat((torch.full((1,), first, device="cuda", dtype=torch.float64),
                       torch.logspace(math.log10(0.003), math.log10(max(rest, 0.0031)), 149, device="cuda", dtype=torch.float64)))
        s = s / s.norm()
        s = s[s >= 0.0025]
        x = (q1[:, :len(s)] * s) @ q2[:len(s)]
        o = T.orthogonalize(x.float()[None])[0].double()
        got = torch.linalg.svdvals(o.cpu())[:len(s)]
        off = tolerance(o[None], 5)
        assert float(got.min()) >= 0.68 - off and float(got.max()) <= MOST + off
