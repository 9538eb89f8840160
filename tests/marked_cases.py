"""Rows whose tokens all count the same - queries of zeros - and whose values mark the 32 tokens that a step of the few-row kernel takes: what is left out or counted twice shows.

The marks: token j's value is 1 in feature j // 32 % D and 0 elsewhere, so a query that sees n tokens has c_f / n times what 1 is kept as in feature f, c_f the number of its tokens with that mark, and
lse = ln n.  Every probability is a power of two, and sums of whole numbers below 2^24 of them are exact in 32 bits: lse is off by a logarithm's last place and two roundings,
2^-20 (1 + lse); out by the quotient's rounding, 2^-22, the result's, u, and where values are made into 16 bits first by another u."""
import math

import torch

from cache_cases import UNIT


def marks(n, D):
    """[n, D]"""
    return torch.nn.functional.one_hot(torch.arange(n) // 32 % D, D).double()


def wanted(sees, D, one):
    """(out [D], lse) of a query that sees so many tokens; one: what a value of 1 is kept as."""
    return marks(sees, D).sum(0) * one / sees, math.log(sees)


def tolerances(out, lse, dtype, roundings):
    return out.abs() * (roundings * UNIT[dtype] + 2.0 ** -22), 2.0 ** -20 * (1 + abs(lse))


def kept_as(dtype, bits):
    """What 1 is kept as beside zeros: itself, or 15 times the least scale of the type that reaches it."""
    if bits == 16:
        return 1.0
    s = torch.tensor(1 / 15, dtype=torch.float64).to(dtype)
    if float(s) * 15 < 1:
        s = (s.view(torch.int16) + 1).view(dtype)
    return float(s) * 15
