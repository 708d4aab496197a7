"""How far linear attention's results in fp32 may be from 64 bits, in norms.

A result is a sum of products.  Each goes through fewer than n = dk + dv + steps + 64 roundings of at most 2^-24 on its way, and so does what has been
added up, which for terms of either sign is about the root of their squares' sum, R.  The roundings' signs are independent, so errors add up as squares:
sqrt(n) 2^-24 R, of which 2 are allowed in the norm over many results.  R comes of the same formulas on squares (the squares of decays are those of
twice their logarithms).  Where inputs are of 16 bits, fp32 operands of a result in fp32 are sums of numbers of 16 bits, off by 2^-22 at most, twice."""
import math

import torch

NAMES = ("y", "last", "dq", "dk", "dv", "dg", "dh0")


def squares(reference, q, k, v, g, h0, n, dy, dlast):
    """R of every result."""
    of = reference(*(x.double().square() for x in (q, k, v)), 2 * g.double(), h0.double().square(), n, dy.double().square(), dlast.double().square())
    return {name: of[name].sqrt() for name in NAMES}


def tolerance(dk, dv, steps, half=False):
    """Of a result's error to R, in norms."""
    return 2 * math.sqrt(dk + dv + steps + 64) * 2.0 ** -24 + (2.0 ** -21 if half else 0.0)
