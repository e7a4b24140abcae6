"""How far fp32 arithmetic may be from 64 bits in a product and in what follows it.

A sum of n products in fp32, in any order, is off by at most about n * 2^-24 of the sum of magnitudes; 2 (n + 8) * 2^-24 covers a
matrix instruction that rounds inside too.  Activations in fp32 are off by 8 * 2^-24 of their value and, where 1 + erf
cancels, of their argument; slopes by 16 * 2^-24 of 1 + their argument's magnitude.  No activation is steeper than 1.13, no slope
changes faster than 1 per unit (what is stored of a pre-activation is the input of the backward pass, so only the forward
pass needs that).  A stored value is rounded once."""
import numpy as np

from oracle import products as op
from tests.operators_harness import EPS, STORED

STEEPEST = 1.13


def summed(a, b, ea=0.0, n=None):
    """Bound of a @ b where a is off by ea."""
    n = a.shape[-1] if n is None else n
    off = 2 * (n + 8) * EPS * (np.abs(a) @ np.abs(b))
    if not np.isscalar(ea):
        off = off + (1 + 2 * (n + 8) * EPS) * (ea @ np.abs(b))
    return off


def act_off(act, v):
    return 0.0 if act == "none" else 8 * EPS * (np.abs(op.activate(act, v)) + np.abs(v))


def slope_off(act, v):
    return 0.0 if act == "none" else 16 * EPS * (1 + np.abs(v))


def stored(dtype, v, off):
    """... and rounded to dtype."""
    return off + STORED[dtype] * (np.abs(v) + off)
