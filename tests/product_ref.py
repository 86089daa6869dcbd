"""How far a product of 32-bit operands in three bf16 parts each may be from 64 bits, in the norm: a bound that does not grow with the contraction as a
worst case does, and so sees the small products that are the difference to fewer parts."""
import numpy as np

from tests.head_ref import EPS32

PAIRS = ((0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0))      # parts of the operands whose products are kept


def norm_bound(k):
    """Of the error's norm over the result's, for operands without a common sign.  The six products are 6 k / 16 additions to a 32-bit sum; each is
    off by 2^-24 / sqrt(3) of the sum in the mean square, which is half of the result's square on the way: 0.25 sqrt(k) 2^-24 together.  Twice
    that for what a matrix instruction rounds within its own sixteen products, and 2^-22 for the output's rounding and the products left out
    (1.7e-3 is what a part leaves of a value: its cube three times)."""
    return 0.5 * k ** 0.5 * EPS32 + 2.0 ** -22


def parts(x):
    """three bf16 parts of 32-bit values, as 64-bit numbers"""
    import torch
    rest, out = torch.as_tensor(x, dtype=torch.float32), []
    for _ in range(3):
        p = rest.bfloat16().float()
        out.append(p.double().numpy())
        rest = rest - p
    return out


def product(x, w, pairs=PAIRS):
    """x w by those products alone, summed in 64 bits"""
    a, b = parts(x), parts(w)
    return sum(np.matmul(a[i], b[j]) for i, j in pairs)


def off(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))
