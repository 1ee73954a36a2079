"""Attention on the GPU against the formula in 64 bits: prompts of many lengths
and single tokens, types, head layouts and sizes, pages, windows, holes, slots
without a sequence, values that are not finite where nobody looks."""

import numpy as np
import pytest

from paper_2110_06037_amd import Attention, KVCache, native as N
from tests.attn_util import Paged, assert_attention, attend, i32
from tests.seq_util import device, host, rounded, strided

pytestmark = pytest.mark.gpu


def run_case(dtype, store, heads, kv, dim, page, lens, past, window=0, seed=0, extra=0, equal=False, size=1.5, scale=None,
             holes=(), step=False, k=None, v=None, max_seqs=None, max_tokens=None):
    """Rows of each sequence against 64 bits; `holes`: (sequence, entry) of the table that are gone."""
    import torch
    r = np.random.default_rng(seed + 1)
    held = [max(0, p + n) for p, n in zip(past, lens)]
    p = Paged(dtype, store, kv, dim, page, held, seed=seed, k=k, v=v)
    for b, i in holes:
        p.table[b, i] = -1
    n = sum(lens)
    q = rounded(r.standard_normal((n, heads * dim)) * size, dtype)
    op = Attention(dtype, heads, kv, dim, page=page, store=store, scale=scale, window=window, max_seqs=max_seqs or len(lens),
                   max_tokens=max_tokens or max(n, 1))
    dq = strided(q, dtype, extra) if extra else device(q, dtype)
    out = torch.full((n, heads * dim + extra), 77.0, dtype=dq.dtype, device="cuda")[:, :heads * dim]
    if step:
        got = host(op.step(dq, p.cache, p.table, i32(past), out=out))
    else:
        got = host(op.run(dq, p.cache, p.table, i32(past), offsets=None if equal else i32(np.concatenate([[0], np.cumsum(lens)])),
                          out=out))
    at = 0
    for b, (m, s) in enumerate(zip(lens, past)):
        rows, at = slice(at, at + m), at + m
        g = got[rows].reshape(m, heads, dim)
        if s < 0:
            assert not g.any()
            continue
        seen = np.ones(s + m, bool)
        for bb, i in holes:
            if bb == b:
                seen[i * page:(i + 1) * page] = False
        y, a, bound = attend(q[rows].reshape(m, heads, dim), *p.rows(b), kv, s, window, seen, scale)
        assert_attention(g, y, a, bound, dtype, f"sequence {b}: {m} rows after {s}")
    return got


LENS, PAST = [70, 0, 1, 33, 200, 64, 2], [0, 5, 0, 16, 31, 1000, 129]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (8, 1, 128), (3, 3, 80)])
def test_prompts(dtype, store, heads, kv, dim):
    run_case(dtype, store, heads, kv, dim, 16, LENS, PAST)
    run_case(dtype, store, heads, kv, dim, 64, [50, 50], [0, 300], equal=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (8, 1, 128), (3, 3, 80)])
def test_tokens(dtype, store, heads, kv, dim):
    run_case(dtype, store, heads, kv, dim, 16, [1] * 9, [0, 1, 15, 16, 62, 63, 64, 777, 2500], step=True)
    run_case(dtype, store, heads, kv, dim, 64, [1], [5000], step=True)


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 64, 72, 88, 96, 104, 112, 120, 128, 136, 160, 192, 200, 224, 248, 256])
@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("bf16", "i8"), ("f32", "same"), ("f16", "i8")])
def test_head_sizes(dim, dtype, store):
    run_case(dtype, store, 4, 2, dim, 32, [75, 3], [0, 90], seed=dim)
    run_case(dtype, store, 4, 2, dim, 32, [1, 1, 1], [0, 200, 77], seed=dim, step=True)


@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (5, 1), (16, 1), (17, 1), (40, 1), (71, 1), (6, 2), (33, 11), (64, 4), (12, 12)])
def test_head_layouts(heads, kv):
    for dtype, store in (("bf16", "same"), ("f16", "i8")):
        run_case(dtype, store, heads, kv, 64, 16, [40, 1, 130], [0, 60, 7])
        run_case(dtype, store, heads, kv, 64, 16, [1, 1, 1], [0, 300, 70], step=True)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
def test_pages(page):
    for dtype, store in (("bf16", "same"), ("f32", "i8"), ("f16", "same")):
        run_case(dtype, store, 4, 2, 64, page, [100, 31, 5], [0, 300, 1023])
        run_case(dtype, store, 4, 2, 64, page, [1, 1, 1], [15, 300, 1023], step=True)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 63, 64, 65, 100, 128, 500, 5000])
def test_windows(window):
    for dtype, store in (("bf16", "same"), ("f32", "same"), ("f16", "i8")):
        run_case(dtype, store, 4, 2, 64, 16, [70, 1, 33, 200], [0, 60, 300, 45], window=window)
        run_case(dtype, store, 4, 2, 64, 16, [1] * 5, [0, 14, 63, 300, 1111], window=window, step=True)


@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("f16", "i8"), ("f32", "same")])
def test_slots_without_a_sequence_and_holes(dtype, store):
    run_case(dtype, store, 4, 2, 64, 16, [5, 40, 3, 70], [-1, 50, -9, 0], holes=[(1, 0), (1, 3), (3, 2)])
    run_case(dtype, store, 4, 2, 64, 16, [1] * 6, [-1, 50, -1, 500, 0, 40], holes=[(1, 0), (1, 3), (3, 0), (3, 31), (4, 0)], step=True)
    # every page of the window gone
    run_case(dtype, store, 4, 2, 64, 16, [4, 1], [100, 100], window=10, holes=[(0, 5), (0, 6), (1, 5), (1, 6)])
    run_case(dtype, store, 4, 2, 64, 16, [1, 1], [100, 100], window=10, holes=[(0, 5), (0, 6), (1, 6)], step=True)


@pytest.mark.parametrize("extra", [1, 4, 8])
def test_strided_and_unaligned_rows(extra):
    for dtype in ("bf16", "f32"):
        run_case(dtype, "same", 4, 2, 64, 16, [50, 9], [0, 20], extra=extra)
        run_case(dtype, "i8", 4, 2, 64, 16, [1, 1], [50, 20], extra=extra, step=True)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales(scale):
    run_case("bf16", "same", 4, 2, 64, 16, [50, 9], [0, 20], scale=scale)
    run_case("f32", "i8", 4, 2, 64, 16, [1, 1], [50, 20], scale=scale, step=True)


@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("f16", "same"), ("f16", "i8"), ("f32", "same")])
def test_sharp_rows(dtype, store):
    # scores of hundreds: one key has nearly all of a row's weight
    run_case(dtype, store, 4, 2, 64, 16, [150], [40], size=60)
    run_case(dtype, store, 4, 2, 64, 16, [1, 1], [1000, 333], size=60, step=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "i8"])
def test_values_that_are_not_finite_stay_where_they_are(dtype, store):
    # rows before a key or value that holds an infinity or a NaN do not see it
    r = np.random.default_rng(5)
    for bad in (np.inf, -np.inf, np.nan):
        for which in (0, 1):
            kv = [rounded(r.standard_normal((150, 128)), dtype) for _ in range(2)]
            kv[which][70, 3], kv[which][101, 100] = bad, bad
            got = run_case(dtype, store, 4, 2, 64, 16, [150], [0], k=kv[0].copy(), v=kv[1].copy()) if which else None
            if which == 0:
                # (what a bad key does to the rows that see it is the softmax's matter)
                p = Paged(dtype, store, 2, 64, 16, [150], k=kv[0].copy(), v=kv[1].copy())
                clean = Paged(dtype, store, 2, 64, 16, [150], k=np.where(np.isfinite(kv[0]), kv[0], 0), v=kv[1].copy())
                q = device(rounded(r.standard_normal((150, 256)), dtype), dtype)
                op = Attention(dtype, 4, 2, 64, page=16, store=store, max_tokens=150)
                a, b = host(op.run(q, p.cache, p.table, i32([0]))), host(op.run(q, clean.cache, clean.table, i32([0])))
                assert np.array_equal(a[:70], b[:70]) and np.array_equal(a[70:101, 128:], b[70:101, 128:])
            # a window that has passed them, for single tokens
            p = Paged(dtype, store, 2, 64, 16, [150], k=kv[0].copy(), v=kv[1].copy())
            op = Attention(dtype, 4, 2, 64, page=16, store=store, window=20)
            q = device(rounded(r.standard_normal((1, 256)), dtype), dtype)
            assert np.isfinite(host(op.step(q, p.cache, p.table, i32([149])))).all()
            assert np.isfinite(host(op.step(q, p.cache, p.table, i32([69])))).all()
            assert np.isfinite(host(op.run(q, p.cache, p.table, i32([149])))).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_a_row_does_not_depend_on_its_neighbours(dtype):
    import torch
    p = Paged(dtype, "same", 2, 64, 16, [300] * 3)
    op = Attention(dtype, 8, 2, 64, page=16, max_seqs=3, max_tokens=300)
    q = torch.randn(300, 512, device="cuda").to(p.cache.torch_dtype)
    bad = q.clone()
    bad[7, 70], bad[40, 500], bad[299] = float("nan"), float("inf"), 1e4
    past = i32([200] * 3)
    a, b = op.run(q, p.cache, p.table, past), op.run(bad, p.cache, p.table, past)
    keep = torch.ones(300, 8, dtype=torch.bool, device="cuda")
    keep[7, 1] = keep[40, 7] = False
    keep[299] = False
    assert torch.equal(a.view(300, 8, 64)[keep], b.view(300, 8, 64)[keep])
    assert torch.isnan(b.view(300, 8, 64)[7, 1]).all()
    a, b = (op.step(t[[6, 7, 8]], p.cache, p.table, past) for t in (q, bad))
    keep = torch.ones(3, 8, dtype=torch.bool, device="cuda")
    keep[1, 1] = False
    assert torch.equal(a.view(3, 8, 64)[keep], b.view(3, 8, 64)[keep]) and torch.isnan(b.view(3, 8, 64)[1, 1]).all()


def test_rows_behind_the_last_sequence_are_left_alone():
    import torch
    p = Paged("bf16", "same", 1, 64, 16, [20, 9])
    op = Attention("bf16", 2, 1, 64, page=16, max_seqs=2, max_tokens=40)
    q, out = torch.randn(40, 128, device="cuda").bfloat16(), torch.full((40, 128), 5.0, device="cuda").bfloat16()
    want = op.run(q[2:31].clone(), p.cache, p.table, i32([0, 0]), offsets=i32([0, 20, 29]))
    op.run(q, p.cache, p.table, i32([0, 0]), offsets=i32([2, 22, 31]), out=out)
    assert torch.equal(out[2:31], want) and (out[:2] == 5).all() and (out[31:] == 5).all()
    # offsets outside the call's rows, and falling ones, lead nowhere else
    for offsets in ([-5, 1 << 30, 1 << 30], [0, 30, 10], [50, 60, 70]):
        op.run(q, p.cache, p.table, i32([0, 0]), offsets=i32(offsets), out=out)
    # and the handle computes as before
    assert torch.equal(op.run(q[2:31].clone(), p.cache, p.table, i32([0, 0]), offsets=i32([0, 20, 29])), want)
    assert op.run(q[:0], p.cache, p.table, i32([0, 0])).shape == (0, 128)


def test_sequences_share_pages():
    import torch
    p = Paged("bf16", "same", 2, 64, 16, [100])
    op = Attention("bf16", 4, 2, 64, page=16, max_seqs=3)
    q = torch.randn(1, 256, device="cuda").bfloat16()
    one = op.step(q, p.cache, p.table, i32([99]))
    three = op.step(q.expand(3, 256).contiguous(), p.cache, p.table.expand(3, -1), i32([99, 99, 99]))
    assert all(torch.equal(one[0], t) for t in three)


def test_repeated_calls_agree():
    # the joining of parts does not depend on which part ends last
    import torch
    p = Paged("bf16", "i8", 2, 128, 16, [4000, 17, 900])
    op = Attention("bf16", 8, 2, 128, page=16, store="i8", max_seqs=3, max_tokens=64)
    q = torch.randn(3, 1024, device="cuda").bfloat16()
    past = i32([3999, 16, 899])
    want = op.step(q, p.cache, p.table, past)
    rows = torch.randn(40, 1024, device="cuda").bfloat16()
    prompt = op.run(rows, p.cache, p.table[:1], i32([3960]))
    for _ in range(20):
        assert torch.equal(op.step(q, p.cache, p.table, past), want)
        assert torch.equal(op.run(rows, p.cache, p.table[:1], i32([3960])), prompt)


def test_overlaps_are_refused():
    import torch
    p = Paged("bf16", "same", 2, 64, 16, [20])
    op = Attention("bf16", 4, 2, 64, page=16, max_tokens=20)
    wide = torch.randn(20, 512, device="cuda").bfloat16()
    inside = p.cache.v.view(-1)[:20 * 256].view(20, 256)
    for out in (wide[:, :256], wide[:, 100:356], inside):
        with pytest.raises(N.SNError) as e:
            op.run(wide[:, :256], p.cache, p.table, i32([0]), out=out)
        assert e.value.code == -1 and "overlaps" in str(e.value)
    want = op.run(wide[:, :256].clone(), p.cache, p.table, i32([0]))
    assert torch.equal(op.run(wide[:, :256], p.cache, p.table, i32([0]), out=wide[:, 256:]), want)
