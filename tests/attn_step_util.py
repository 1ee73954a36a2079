"""The bound of single tokens over a cache, whose weights keep more bits than a prompt's.

In the terms of ``attn_util`` (A = sum p |v| / sum p, u the unit roundoff of the type), derived
before any run: the result's rounding, u |y|; the float32 part, ``attend``'s third value; and
what the step's weights lose before they meet v, in place of a prompt's 2 u A:

* float32: nothing;
* two bf16 parts (bf16, and 8-bit caches of 16-bit types): the first is off by at most 2^-8
  of the weight, which the second holds but for 2^-8 of it: 2^-16 A.  Codes of 8 bits are
  exact in bf16, and values of a cache in dtype are operands as they are;
* f16 once (caches in f16): 2^-11 A; and weights, which are stored 2^14 times as large, below
  2^-28 of the largest round to multiples of 2^-24 2^-14, half of which, 2^-39, may be lost of
  each, of |v| at most its largest; sum p is at least the largest weight, 1."""

import numpy as np

from tests.seq_util import FLOOR, UNIT


def step_limit(dtype, store, y, a, bound, v, seen):
    """How far an output may be off; v: the values seen, `seen` keys."""
    u = UNIT[dtype]
    if dtype == "f32":
        rough = 0.0
    elif dtype == "bf16" or store == "i8":
        rough = 2.0 ** -16 * a
    else:
        rough = 2.0 ** -11 * a + seen * 2.0 ** -39 * np.abs(v).max(initial=0)
    return u * np.abs(y) + (1 + u) * (rough + bound) + FLOOR[dtype]


def times_the_limit(got, y, limit):
    return float((np.abs(got - y) / limit).max(initial=0))
