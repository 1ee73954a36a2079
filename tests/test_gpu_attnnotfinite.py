"""Attention on the GPU over values and scores that are not finite, against the formula's limit:
every seen key has a weight above zero, however small, so a seen infinity is the
result's, a NaN or infinities of both signs are NaN, wherever the row's tile, part or call ends."""

import numpy as np
import pytest

from paper_2110_06037_amd import Attention
from tests.attn_util import Paged, assert_attention, attend, i32
from tests.seq_util import device, host, rounded

pytestmark = pytest.mark.gpu
N, DIM, KV, HEADS, PAGE = 700, 64, 2, 6, 16
# (position, key head, element, value)
BAD = [(20, 0, 3, np.inf), (40, 0, 9, -np.inf), (30, 0, 11, np.nan), (21, 0, 13, np.inf), (333, 0, 13, -np.inf), (130, 1, 63, np.inf),
       (131, 1, 62, -np.inf), (400, 1, 0, np.nan), (401, 1, 1, np.inf), (402, 1, 1, np.inf), (600, 0, 5, -np.inf)]


def classes(v, past, n, window, seen):
    """The values that are not finite as the rows [n, kv, dim] see them: 0 where none is."""
    out = np.zeros((n, *v.shape[1:]))
    for i in range(n):
        at = np.arange(len(v))
        see = (at <= past + i) & (at > past + i - window if window else True) & seen
        with np.errstate(invalid="ignore"):
            bad = v[see]
            out[i] = np.where(np.isfinite(bad), 0, bad).sum(0)
    return out


def check(got, q, k, v, past, dtype, window, seen, what):
    n = len(q)
    bad = np.repeat(classes(v, past, n, window, seen), HEADS // KV, 1)
    y, a, bound = attend(q, k, np.where(np.isfinite(v), v, 0), KV, past, window, seen)
    # the finite elements as ever, the others by their class
    assert np.array_equal(got[bad != 0], bad[bad != 0], equal_nan=True), f"{what}: other classes"
    assert np.isfinite(got[bad == 0]).all(), what
    assert_attention(np.where(bad == 0, got, 0), np.where(bad == 0, y, 0), a, bound, dtype, what)


def problem(dtype, gap, big, seed=0):
    """Scores about 0, but `gap` octaves more at the keys `big`."""
    r = np.random.default_rng(seed)
    k, v = r.standard_normal((N, KV, DIM)) * 0.25, r.standard_normal((N, KV, DIM))
    q = r.standard_normal((N, HEADS, DIM))
    k[:, :, 0], q[:, :, 0] = 0, 8
    k[big, :, 0] = gap * np.log(2)
    for at, head, d, value in BAD:
        v[at, head, d] = value
    return (rounded(t.reshape(N, -1), dtype) for t in (q, k, v))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap", [0, 30, 60, 600])
@pytest.mark.parametrize("big", [[2], [690], [2, 350]])
@pytest.mark.parametrize("window", [0, 150])
def test_a_seen_infinity_counts_whatever_its_weight(dtype, gap, big, window):
    q, k, v = problem(dtype, gap, big)
    p = Paged(dtype, "same", KV, DIM, PAGE, [N], k=k.copy(), v=v.copy())
    q, k, v = q.reshape(N, HEADS, DIM), k.reshape(N, KV, DIM), v.reshape(N, KV, DIM)
    hole = np.ones(N, bool)
    p.table[0, 2], hole[32:48] = -1, False
    narrow = Attention(dtype, HEADS, KV, DIM, page=PAGE, window=window, max_seqs=40, max_tokens=N)
    wide = p.table.new_full((1, 4000), -1)  # (many parts)
    wide[:, :p.table.shape[1]] = p.table

    def rows(a, b):
        return device(q[a:b].reshape(b - a, -1), dtype)

    # one row meets many tiles, places in them and parts
    for table in (p.table, wide):
        for a, b in ((0, N), (0, 64), (65, 128), (100, 141), (128, 400), (350, 353), (640, N), (N - 1, N)):
            got = host(narrow.run(rows(a, b), p.cache, table, i32([a]))).reshape(b - a, HEADS, DIM)
            check(got, q[a:b], k[:b], v[:b], a, dtype, window, hole[:b], f"rows {a} to {b}, table of {table.shape[1]}")
    at = np.array([0, 19, 20, 21, 29, 30, 39, 40, 63, 64, 129, 130, 131, 180, 332, 333, 399, 400, 401, 402, 483, 599, 600, 689, 690, N - 1])
    for table in (p.table, wide):
        got = host(narrow.step(device(q[at].reshape(len(at), -1), dtype), p.cache, table.expand(len(at), -1), i32(at)))
        for i, past in enumerate(at):
            check(got[i].reshape(1, HEADS, DIM), q[past:past + 1], k[:past + 1], v[:past + 1], past, dtype, window, hole[:past + 1],
                  f"step at {past}, table of {table.shape[1]}")
            one = host(narrow.step(rows(past, past + 1), p.cache, table, i32([past])))
            check(one.reshape(1, HEADS, DIM), q[past:past + 1], k[:past + 1], v[:past + 1], past, dtype, window, hole[:past + 1],
                  f"single step at {past}, table of {table.shape[1]}")


@pytest.mark.parametrize("dtype,dim", [("bf16", 72), ("f16", 96), ("f32", 128), ("bf16", 256), ("f32", 200), ("f16", 8)])
def test_other_sizes(dtype, dim):
    # an infinity in the last element and one in the first, in prompts whole, in parts and in steps
    r = np.random.default_rng(dim)
    n, kv = 200, 2
    q, k, v = (rounded(r.standard_normal((n, kv * dim)), dtype) for _ in range(3))
    v[3, dim - 1], v[77, dim], v[150, 2 * dim - 1], v[150, 0] = np.inf, -np.inf, np.nan, np.inf
    p = Paged(dtype, "same", kv, dim, 16, [n], k=k.copy(), v=v.copy())
    wide = p.table.new_full((1, 3000), -1)
    wide[:, :p.table.shape[1]] = p.table
    op = Attention(dtype, kv, kv, dim, page=16, max_seqs=n, max_tokens=n)
    with np.errstate(invalid="ignore"):
        want = np.stack([np.where(np.isfinite(v[:i + 1]), 0, v[:i + 1]).sum(0) for i in range(n)])
    dq = device(q, dtype)
    for got in (op.run(dq, p.cache, p.table, i32([0])), op.run(dq, p.cache, wide, i32([0])),
                op.step(dq, p.cache, p.table.expand(n, -1), i32(np.arange(n)))):
        got = host(got)
        assert np.array_equal(got[want != 0], want[want != 0], equal_nan=True) and np.isfinite(got[want == 0]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_in_8_bits_that_are_not_finite(dtype):
    # a row with an infinity or a NaN stands for NaN: in all elements of its key head
    q, k, v = problem(dtype, 600, [2])
    p = Paged(dtype, "i8", KV, DIM, PAGE, [N], k=k.copy(), v=v.copy())
    op = Attention(dtype, HEADS, KV, DIM, page=PAGE, store="i8", max_seqs=N, max_tokens=N)
    first = [min(at for at, head, _, _ in BAD if head == h) for h in range(KV)]
    for got in (op.run(device(q, dtype), p.cache, p.table, i32([0])),
                op.step(device(q, dtype), p.cache, p.table.expand(N, -1), i32(np.arange(N)))):
        got = host(got).reshape(N, KV, -1)
        for h in range(KV):
            assert np.isfinite(got[:first[h], h]).all() and np.isnan(got[first[h]:, h]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_scores_of_minus_infinity(dtype, window):
    # such a key has no weight; a row that sees no others has 0 / 0
    r = np.random.default_rng(1)
    q, k, v = (rounded(r.standard_normal((N, m * DIM)), dtype) for m in (HEADS, KV, KV))
    q, k = q.reshape(N, HEADS, DIM), k.reshape(N, KV, DIM)
    q[:, :, 0] = 1
    off = np.zeros(N, bool)
    off[:3] = off[100:180] = off[256:320] = True
    k[off, :, 0] = -np.inf
    p = Paged(dtype, "same", KV, DIM, PAGE, [N], k=k.reshape(N, -1).copy(), v=v.copy())
    wide = p.table.new_full((1, 4000), -1)
    wide[:, :p.table.shape[1]] = p.table
    v = v.reshape(N, KV, DIM)
    at = np.arange(N)
    see = (at <= at[:, None]) & (at > at[:, None] - window if window else True)
    void = ~(see & ~off).any(1)
    # (the same with keys that are finite and not seen)
    y, a, bound = attend(q, np.where(off[:, None, None], 0, k), v, KV, 0, window, ~off)
    op = Attention(dtype, HEADS, KV, DIM, page=PAGE, window=window, max_seqs=N, max_tokens=N)
    flat = q.reshape(N, -1)
    outs = {"prompt": op.run(device(flat, dtype), p.cache, p.table, i32([0])),
            "parts": op.run(device(flat, dtype), p.cache, wide, i32([0])),
            "steps": op.step(device(flat, dtype), p.cache, p.table.expand(N, -1), i32(at)),
            "few rows": None}
    import torch
    cuts = [0, 1, 2, 5, 90, 110, 130, 179, 181, 250, 300, 319, 321, 500, N]
    outs["few rows"] = torch.cat([op.run(device(flat[i:j], dtype), p.cache, wide, i32([i])) for i, j in zip(cuts, cuts[1:])])
    outs["single steps"] = torch.cat([op.step(device(flat[i:i + 1], dtype), p.cache, p.table, i32([i])) for i in range(N)])
    for what, got in outs.items():
        got = host(got).reshape(N, HEADS, DIM)
        assert np.isnan(got[void]).all(), f"{what}: rows without a weight"
        assert_attention(got[~void], y[~void], a[~void], bound[~void], dtype, what)
    # places that do not exist and slots without a sequence are not seen: zeros, as ever
    p.table[0, :7] = -1
    got = host(op.step(device(flat[[2, 50, 99]], dtype), p.cache, p.table.expand(3, -1), i32([2, 50, -1])))
    assert not got.any()
    assert not host(op.run(device(flat[:100], dtype), p.cache, p.table, i32([0]))).any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "i8"])
def test_queries_that_are_not_finite(dtype, store):
    # an infinite element against keys of one sign: all scores minus infinity, 0 / 0, or all plus infinity;
    # other heads and rows as ever
    r = np.random.default_rng(2)
    n = 150
    q, k, v = (rounded(r.standard_normal((n, m * DIM)), dtype) for m in (HEADS, KV, KV))
    q, k = q.reshape(n, HEADS, DIM), k.reshape(n, KV, DIM)
    k[:, :, 0] = rounded(-np.abs(k[:, :, 0]) - 1, dtype)
    clean = q.copy()
    q[::3, 1, 0], q[1::3, 4, 0] = np.inf, -np.inf
    bad = ~np.isfinite(q).all(-1)
    p = Paged(dtype, store, KV, DIM, PAGE, [n], k=k.reshape(n, -1).copy(), v=v.copy())
    wide = p.table.new_full((1, 4000), -1)
    wide[:, :p.table.shape[1]] = p.table
    op = Attention(dtype, HEADS, KV, DIM, page=PAGE, store=store, max_seqs=n, max_tokens=n)

    def outs(q):
        d = device(q.reshape(n, -1), dtype)
        yield op.run(d, p.cache, p.table, i32([0]))
        yield op.run(d, p.cache, wide, i32([0]))
        yield op.step(d, p.cache, p.table.expand(n, -1), i32(np.arange(n)))

    for got, want in zip(outs(q), outs(clean)):
        got, want = host(got).reshape(n, HEADS, DIM), host(want).reshape(n, HEADS, DIM)
        assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad]) and np.isfinite(want).all()
