"""What long sums in fp32 may be off in the 2-norm over many results.

An addition's rounding is at most U = 2^-24 of the sum so far and spread evenly over both sides: U / sqrt(3) of it in the root mean
square.  Of terms that are independent and of one size the sum's square grows evenly, so that a chain of m additions out of n terms
puts in m^2 / (2 n) of the result's square times U^2 / 3, and the n / m chains of a result m U^2 / 6."""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def off(got, exact):
    return float((got.double() - exact).norm() / exact.norm())


def bound(terms, dtype, folded=0, parts=1):
    """folded: terms that are added up by themselves before their sum is (0: all); parts: of a sum that is divided, at most.  The
    last rounding, to dtype, is of the same kind."""
    chain = terms if not folded else min(terms, folded) + -(-terms // folded)
    return math.sqrt((chain + parts - 1) / 6 * U ** 2 + HALF_STEP[dtype] ** 2 / 3)
