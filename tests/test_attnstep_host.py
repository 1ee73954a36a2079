"""The steps' bound on the CPU: outputs whose weights keep what the kernel promises lie within
it, those with fewer bits, or without a key, do not."""

import numpy as np
import pytest

from tests.attn_step_util import step_limit, times_the_limit
from tests.attn_util import attend
from tests.seq_util import rounded

KV, DIM = 16, 64


def simulated(keys, weights, drop=None):
    """One token over `keys` keys in bf16, its weights through `weights`: how far off, in limits."""
    r = np.random.default_rng(keys)
    q = rounded(r.standard_normal((1, KV, DIM)) * 1.5, "bf16")
    k, v = (rounded(r.standard_normal((keys, KV, DIM)), "bf16") for _ in range(2))
    y, a, bound = attend(q, k, v, KV, keys - 1, 0)
    got = np.zeros_like(y)
    for h in range(KV):
        s = k[:, h] @ q[0, h] * DIM ** -0.5
        p = np.exp(s - s.max()).astype(np.float32).astype(np.float64)
        w = weights(p)
        if drop is not None:
            w[drop] = 0
        got[0, h] = w @ v[:, h] / p.sum()
    return times_the_limit(rounded(got, "bf16"), y, step_limit("bf16", "same", y, a, bound, v, keys))


def two_parts(p):
    high = rounded(p, "bf16")
    return high + rounded(p - high, "bf16")


@pytest.mark.parametrize("keys", [16, 64, 777, 2501])
def test_the_bound_holds_for_two_parts(keys):
    assert simulated(keys, two_parts) <= 1


# Weights of 8 bits are off by about 2^-9 each, an output by 2^-9 A / sqrt(keys) where they are
# alike, the largest of a thousand outputs by three times that; the bound's float32 sums are worth
# 2 keys 2^-24 A in the worst case, which is more from (3 2^14)^(2 / 3) = 1340 keys on.
@pytest.mark.parametrize("keys", [16, 64, 777])
def test_the_bound_tells_weights_apart(keys):
    assert simulated(keys, lambda p: rounded(p, "bf16")) > 1
    # the second part with the wrong sign
    assert simulated(keys, lambda p: 2 * rounded(p, "bf16") - two_parts(p)) > 1
    assert simulated(keys, two_parts, drop=keys // 2) > 1
