"""Helpers of the sequence operators' tests: tensors of an element type, and
the bound of a result's error against 64 bits.

Tolerances, derived before any run.  An output of type T is one rounding of a
float32 value: at most u(T) of its size, the unit roundoff 2^-p of p
significant bits: 2^-8 (bf16), 2^-11 (f16), 2^-24 (f32).  The float32 value itself is
a sum of n products with errors of at most about n * 2^-24 of the sum of the
products' sizes; hardware exp2, reciprocal and square root add a few 2^-23.
So each element may be off by u * |exact| + c * 2^-24 * size, with `size` the
sum of the sizes of what is added up for that element and c a small count of
roundings per term that each test names.  f16 results below 2^-14 round to
multiples of 2^-24: half of that is added."""

import numpy as np

UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FLOOR = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def torch_type(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def rounded(a, dtype):
    """The float64 array's values as the element type holds them."""
    import torch
    return torch.from_numpy(np.asarray(a, np.float64)).to(torch_type(dtype)).double().numpy()


def device(a, dtype):
    """A device tensor of the array's values (given as the type holds them)."""
    import torch
    return torch.from_numpy(np.asarray(a, np.float64)).to(torch_type(dtype)).cuda()


def strided(a, dtype, extra):
    """The same as rows of a wider tensor: `extra` elements before and after each."""
    import torch
    t = device(a, dtype)
    wide = torch.full((t.shape[0], t.shape[1] + 2 * extra), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, extra:extra + t.shape[1]] = t
    return wide[:, extra:extra + t.shape[1]]


def host(t):
    return t.detach().double().cpu().numpy()


def assert_close(got, exact, size, dtype, count, what=""):
    """|got - exact| <= u |exact| + count 2^-24 size, elementwise; the same
    infinities and NaN."""
    got = host(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == exact.shape, (what, got.shape, exact.shape)
    fine = np.isfinite(exact)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: other values are finite"
    limit = UNIT[dtype] * np.abs(exact) + (1 + UNIT[dtype]) * count * 2.0 ** -24 * size + FLOOR[dtype]
    over = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, exact, 0)) / limit, 0)
    assert over.size == 0 or over.max() <= 1, f"{what}: {over.max()} times the bound at {np.unravel_index(over.argmax(), over.shape)}"
