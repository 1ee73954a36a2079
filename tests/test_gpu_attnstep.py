"""Single tokens on the GPU against 64 bits, under the bound of the bits that their weights keep."""

import numpy as np
import pytest

from paper_2110_06037_amd import Attention
from tests.attn_step_util import step_limit, times_the_limit
from tests.attn_util import Paged, attend, i32
from tests.seq_util import device, host, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads,kv,dim", [(8, 8, 64), (16, 2, 128), (6, 3, 80), (4, 2, 256)])
def test_steps_keep_their_weights_bits(dtype, store, heads, kv, dim):
    r = np.random.default_rng(dim)
    past = [0, 1, 15, 63, 64, 300, 776, 2500]
    p = Paged(dtype, store, kv, dim, 16, [n + 1 for n in past], seed=dim)
    q = rounded(r.standard_normal((len(past), heads * dim)) * 1.5, dtype)
    for window in (0, 200):
        op = Attention(dtype, heads, kv, dim, page=16, store=store, window=window, max_seqs=len(past))
        dq = device(q, dtype)
        got = host(op.step(dq, p.cache, p.table, i32(past))).reshape(len(past), 1, heads, dim)
        for b, n in enumerate(past):
            k, v = p.rows(b)
            y, a, bound = attend(q[b].reshape(1, heads, dim), k, v, kv, n, window)
            limit = step_limit(dtype, store, y, a, bound, v, min(n + 1, window or n + 1))
            assert times_the_limit(got[b], y, limit) <= 1, f"{n} keys before, window {window}"
            # and a sequence by itself, in other parts
            one = host(op.step(dq[b:b + 1], p.cache, p.table[b:b + 1], i32([n]))).reshape(1, heads, dim)
            assert times_the_limit(one, y, limit) <= 1, f"{n} keys before, alone, window {window}"
