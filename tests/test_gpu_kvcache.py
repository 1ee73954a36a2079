"""KVCache on the GPU: rows come back as they were, or exactly as their 8-bit
codes stand for; places, pages and slots that do not exist; packed rows of many
lengths; what a write leaves alone."""

import numpy as np
import pytest

from paper_2110_06037_amd import KVCache, native as N
from tests.attn_util import Paged, i32, poison, quantised
from tests.seq_util import device, host, rounded, strided

pytestmark = pytest.mark.gpu


def check(dtype, store, kv, dim, page, lens, past, seed=0, extra=0, equal=False):
    import torch
    r = np.random.default_rng(seed)
    held = [p + n for p, n in zip(past, lens)]
    p = Paged(dtype, store, kv, dim, page, held, seed=seed)
    before = [host(t) for t in p.cache.read(p.table, i32([0] * len(held)), sum(held), offsets=i32(p.starts))]
    n = sum(lens)
    new = [rounded(r.standard_normal((n, kv * dim)) * 3, dtype) for _ in range(2)]
    offsets = None if equal else i32(np.concatenate([[0], np.cumsum(lens)]))
    put = (lambda a: strided(a, dtype, extra)) if extra else (lambda a: device(a, dtype))
    p.cache.write(put(new[0]), put(new[1]), p.table, i32(past), offsets=offsets)
    got = [host(t) for t in p.cache.read(p.table, i32(past), n, offsets=offsets)]
    after = [host(t) for t in p.cache.read(p.table, i32([0] * len(held)), sum(held), offsets=i32(p.starts))]
    at = np.concatenate([np.arange(s + q, s + q + m) for s, q, m in zip(p.starts, past, lens)]).astype(int)
    for old, x, g, a, kept in zip(before, new, got, after, (p.k, p.v)):
        # what the rows stand for, rounded once to dtype (exact codes: no tolerance)
        want = rounded(quantised(x, kv) if store == "i8" else x, dtype)
        assert np.array_equal(old, rounded(kept.reshape(old.shape), dtype))
        assert np.array_equal(g, want)
        old[at] = want
        assert np.array_equal(a, old)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "i8"])
def test_rows_come_back(dtype, store):
    check(dtype, store, 2, 64, 16, [40, 0, 1, 17, 100, 3], [0, 5, 0, 16, 31, 1])
    check(dtype, store, 3, 80, 64, [1, 1, 1, 1], [0, 63, 64, 200], equal=True)
    check(dtype, store, 1, 128, 256, [300, 300], [0, 7], equal=True)


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 72, 96, 120, 136, 192, 248, 256])
@pytest.mark.parametrize("store", ["same", "i8"])
def test_head_sizes(dim, store):
    for dtype in ("bf16", "f32"):
        check(dtype, store, 2, dim, 32, [50, 1, 30], [9, 31, 0], seed=dim)


@pytest.mark.parametrize("extra", [1, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_unaligned_rows(dtype, extra):
    for store in ("same", "i8"):
        check(dtype, store, 2, 64, 16, [33, 20], [0, 15], extra=extra)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_codes_at_the_middle_between_two(dtype):
    # rows whose values lie on and beside the middles of the steps of their scale
    r = np.random.default_rng(3)
    rows = []
    for most in (127.0, 1.0, 254.0, 3.0, 1.984375, 100.0):
        s = float(np.float32(most) * np.float32(1 / 127))
        x = (r.integers(-127, 127, (16, 64)) + 0.5) * s
        x[:, 0] = most
        rows.append(np.where(r.random(x.shape) < 0.5, x, np.nextafter(x.astype(np.float32), np.float32(r.choice([-1e9, 1e9])))))
    x = rounded(np.clip(np.concatenate(rows), -1e4, 1e4), dtype)
    p = Paged(dtype, "i8", 1, 64, 16, [len(x)], k=x, v=x[::-1].copy())
    k, v = p.cache.read(p.table, i32([0]), len(x))
    assert np.array_equal(host(k), rounded(quantised(x, 1), dtype)) and np.array_equal(host(v), host(k)[::-1])


def test_rows_of_zeros_tiny_values_and_values_that_are_not_finite():
    x = np.zeros((6, 128))
    x[1] = 2.0 ** -130
    x[2] = np.linspace(-1, 1, 128) * 2.0 ** -112
    x[3, 5], x[4, 100] = np.inf, np.nan
    x[5] = np.linspace(-3, 3, 128) * 2.0 ** 120
    x = rounded(x, "f32")
    p = Paged("f32", "i8", 2, 64, 16, [6], k=x, v=x)
    for t in p.cache.read(p.table, i32([0]), 6):
        assert np.array_equal(host(t), rounded(quantised(x, 2), "f32"), equal_nan=True)
    same = Paged("f32", "same", 2, 64, 16, [6], k=x, v=x)
    assert np.array_equal(host(same.cache.read(same.table, i32([0]), 6)[1]), x, equal_nan=True)


@pytest.mark.parametrize("store", ["same", "i8"])
def test_places_that_do_not_exist(store):
    import torch
    r = np.random.default_rng(0)
    cache = KVCache("bf16", 2, 64, 6, page=16, store=store)
    poison(cache)
    whole = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    # a hole, an entry beyond the pages, the end of the table, a slot without a
    # sequence, positions near 2^31
    table = i32([[0, -1, 1], [2, 6, 1 << 30], [3, 4, 5], [5, 5, 5], [-7, 2, 2]])
    past = i32([10, 0, 40, -1, (1 << 31) - 1])
    n = 30
    x = [rounded(r.standard_normal((5 * n, 128)), "bf16") for _ in range(2)]
    cache.write(device(x[0], "bf16"), device(x[1], "bf16"), table, past)
    want = [rounded(quantised(t, 2), "bf16") if store == "i8" else t.copy() for t in x]
    pos = np.concatenate([p + np.arange(n) for p in (10, 0, 40, -10 ** 6, 2 ** 31 - 1)])
    ids = np.concatenate([np.where((pos[b * n:(b + 1) * n] >= 0) & (pos[b * n:(b + 1) * n] < 48), np.array(row)[np.clip(
        pos[b * n:(b + 1) * n], 0, 47) // 16], -1) for b, row in enumerate(table.cpu().numpy())])
    there = (ids >= 0) & (ids < 6)
    for w, got in zip(want, cache.read(table, past, 5 * n)):
        w[~there] = 0
        assert np.array_equal(host(got), w)
    # pages that nothing was written to are as they were
    untouched = sorted(set(range(6)) - set(ids[there]))
    assert untouched
    for t, old in zip((t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None), whole):
        assert torch.equal(t[untouched].view(torch.uint8), old[untouched].view(torch.uint8))


def test_rows_behind_the_last_sequence_are_left_alone():
    import torch
    p = Paged("f16", "same", 1, 64, 16, [20, 9])
    k, v = (torch.full((40, 64), 5.0, device="cuda").half() for _ in range(2))
    p.cache.read(p.table, i32([0, 0]), 40, offsets=i32([2, 22, 31]), k_out=k, v_out=v)
    assert np.array_equal(host(k[2:31]), p.k.reshape(29, 64)) and (k[:2] == 5).all() and (v[31:] == 5).all()
    before = p.cache.k.clone()
    p.cache.write(k, v, p.table, i32([0, 0]), offsets=i32([0, 0, 0]))  # no rows of any sequence
    assert torch.equal(torch.nan_to_num(p.cache.k), torch.nan_to_num(before))
    # offsets outside the call's rows lead nowhere else
    p.cache.read(p.table, i32([0, 0]), 40, offsets=i32([-5, 1 << 30, 1 << 30]), k_out=k, v_out=v)
    assert p.cache.read(p.table, i32([0, 0]), 0)[0].shape == (0, 64)


def test_an_empty_cache_holds_nothing():
    import torch
    cache = KVCache("bf16", 1, 64, 0)
    x = torch.ones(3, 64, device="cuda").bfloat16()
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    cache.write(x, x, table, i32([0]))
    assert not cache.read(table, i32([0]), 3)[0].any()
    none = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    assert not KVCache("bf16", 1, 64, 2).read(none, i32([0]), 3)[0].any()


def test_overlaps_are_refused():
    import torch
    p = Paged("bf16", "same", 2, 64, 16, [20])
    flat = p.cache.k.view(-1)
    rows, other = flat[:20 * 128].view(20, 128), torch.zeros(20, 128, device="cuda").bfloat16()
    for f in (lambda: p.cache.write(rows, other, p.table, i32([0])), lambda: p.cache.write(other, rows, p.table, i32([0])),
              lambda: p.cache.read(p.table, i32([0]), 20, k_out=rows, v_out=other),
              lambda: p.cache.read(p.table, i32([0]), 20, k_out=other, v_out=other)):
        with pytest.raises(N.SNError) as e:
            f()
        assert e.value.code == -1 and "overlaps" in str(e.value)
