"""The iteration X <- a X + (b P + c P^2) X, P = X X^T, in 64 bits, and how far a result of fp32 accuracy may be from it."""
import math

import torch

A, B, C = 3.4445, -4.7750, 2.0315
MOST = 1.21             # of a singular value after any iteration: the polynomial's largest in [0, 1] is 1.2024, and it maps [0, 1.21] into itself
SLOPE = 4.25            # of the polynomial in [0, 1.21]; it and the polynomial over its argument bound what becomes of an error, in the Frobenius norm


def iterate(u, iterations, operand=None):
    """In 64 bits; `operand` rounds what enters a product."""
    operand = operand or (lambda x: x)
    u = u.double()
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    norm = x.square().sum((1, 2), keepdim=True).sqrt()
    x = torch.where(norm > 0, x / norm, torch.zeros_like(x))
    for _ in range(iterations):
        x = operand(x)
        p = operand(x @ x.transpose(1, 2).contiguous())
        q = operand(B * p + C * (p @ p) + A * torch.eye(x.shape[1], dtype=torch.float64, device=x.device))
        x = q @ x
    return x.transpose(1, 2) if tall else x


def tolerance(exact, iterations, begin=2.0 ** -22):
    """Of each matrix' error in the Frobenius norm.

    A product L R of operands as two fp16 numbers: an entry of each is off by 2^-22 of it at most, and as much is left out with the product of the two low
    numbers, so 3 2^-22 |L|_F |R|_2 in all.  Its K additions are off by 2^-24 of what has been added up, whose norm is no larger; their signs are
    independent, so sqrt(K) 2^-24.  With u their sum, |X|_2 <= 1.21, |P|_2 <= 1.46, |Q|_2 <= 3.45:
      P   1.21 u |X|_F
      Q   |b| times that, c (2 1.46) times that, c 1.46 u |P|_F, and for its own rounding 2^-22 (3.45 on the diagonal, |b P + c P^2|_F <= 9.4 |X|_F beside it)
      X'  1.21 times Q's, 3.45 u |X|_F, and 2^-22 for what is held of it
    and from one iteration to the next SLOPE times the error.  `begin`: of the first X, relative.  |X_i|_F is that of the exact iteration, for which
    3.4445^i and 1.21 sqrt(shorter side) stand."""
    rows, cols = exact.shape[1:]
    a, b = min(rows, cols), max(rows, cols)
    u_a, u_b = (3 * 2.0 ** -22 + math.sqrt(k) * 2.0 ** -24 for k in (a, b))
    of_p = MOST * u_b
    of_q = (abs(B) + C * 2 * MOST ** 2) * of_p + C * MOST ** 2 * u_a * MOST
    each = MOST * of_q + 3.45 * u_a + 2.0 ** -22 * (3.45 + MOST * 9.4 + 1)
    total = begin * SLOPE ** iterations
    for i in range(iterations):
        total += each * min(A ** i, MOST * math.sqrt(a)) * SLOPE ** (iterations - 1 - i)
    return total


def matrices(shape, seed=1, dtype=torch.float32, scale=0.01, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    n, rows, cols = shape
    rank = max(1, min(rows, cols) // 8)
    x = torch.empty(shape, device=device).normal_(0.0, 1.0, generator=gen)
    x += torch.bmm(torch.empty((n, rows, rank), device=device).normal_(0.0, 2.0, generator=gen),
                   torch.empty((n, rank, cols), device=device).normal_(0.0, 1.0, generator=gen))
    return (x * scale).to(dtype)
