"""What the attention operators' kernels do for large calls, at small cost: more
sequences than a wave looks at, parts that hold several sequences and sequences in
several parts, more tiles than are split, caches beyond 2^32 bytes, other streams,
captured calls, calls on another stream's tensors."""

import numpy as np
import pytest

from paper_2110_06037_amd import Attention, HeadNorm, KVCache
from tests.attn_util import Paged, assert_attention, attend, i32
from tests.seq_util import device, host, rounded
from tests.test_gpu_attention import run_case
from tests.test_gpu_kvcache import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("seqs", [63, 64, 65, 130, 400])
def test_many_sequences(store, seqs):
    r = np.random.default_rng(seqs)
    past = [int(n) for n in r.integers(-1, 150, seqs)]
    run_case("bf16", store, 4, 2, 16, 16, [1] * seqs, past, step=True, seed=seqs)
    lens = [int(n) for n in r.integers(0, 9, seqs)]
    run_case("f16", store, 4, 2, 16, 16, lens, [max(0, p) for p in past], seed=seqs)
    check("bf16", store, 2, 16, 16, lens, [max(0, p) for p in past], seed=seqs)


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_that_hold_several_sequences(dtype, store):
    # 64 key heads leave few workgroups for each: their parts begin and end inside sequences
    r = np.random.default_rng(2)
    for past in ([2000, 3, 0, 700, 64, -1, 128, 1500, 31], [int(n) for n in r.integers(0, 300, 90)], [5000], [63] * 20):
        run_case(dtype, store, 64, 64, 8, 16, [1] * len(past), past, step=True)
        run_case(dtype, store, 64, 64, 8, 16, [1] * len(past), past, step=True, window=100)
    # and with one key head a long sequence is in many parts
    run_case(dtype, store, 17, 1, 8, 16, [1, 1, 1], [60000, 7, 2500], step=True)


@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("f16", "i8"), ("f32", "same")])
def test_more_tiles_than_are_split(dtype, store):
    run_case(dtype, store, 64, 64, 8, 16, [700, 3, 129], [0, 50, 64])
    run_case(dtype, store, 300, 300, 8, 32, [200], [0])


@pytest.mark.parametrize("page", [16, 64])
def test_long_prompts_after_long_pasts(page):
    for dtype, store in (("bf16", "same"), ("bf16", "i8"), ("f32", "i8")):
        run_case(dtype, store, 2, 1, 128, page, [300], [5000])
        run_case(dtype, store, 8, 1, 64, page, [33, 5], [3000, 4097])


@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("f32", "same"), ("f16", "i8")])
def test_caches_beyond_32_bits(dtype, store):
    # K and V of more than 2^32 bytes each, used at their far end
    import torch
    kv, dim, page = 8, 128, 1024
    e = {"bf16": 2, "f32": 4, "f16": 1}[dtype]
    pages = (1 << 32) // (kv * dim * page * e) + 40
    cache = KVCache(dtype, kv, dim, pages, page=page, store=store)
    assert cache.k.numel() * cache.k.element_size() > 1 << 32
    table, past = i32([[pages - 1, pages - 30]]), i32([0])
    r = np.random.default_rng(3)
    k, v = (rounded(r.standard_normal((1100, kv * dim)), dtype) for _ in range(2))
    cache.write(device(k, dtype), device(v, dtype), table, past)
    back = [host(t) for t in cache.read(table, past, 1100)]
    if store == "same":
        assert np.array_equal(back[0], k) and np.array_equal(back[1], v)
    small = KVCache(dtype, kv, dim, 2, page=page, store=store)
    near = i32([[0, 1]])
    small.write(device(k, dtype), device(v, dtype), near, past)
    assert all(np.array_equal(a, host(b)) for a, b in zip(back, small.read(near, past, 1100)))
    op = Attention(dtype, 8, kv, dim, page=page, store=store, max_tokens=60)
    q = device(rounded(r.standard_normal((60, 8 * dim)), dtype), dtype)
    assert torch.equal(op.run(q, cache, table, i32([1040])), op.run(q, small, near, i32([1040])))
    assert torch.equal(op.step(q[:1], cache, table, i32([1099])), op.step(q[:1], small, near, i32([1099])))


def head_norm():
    import torch
    op = HeadNorm("bf16", 8, 2, 64)
    q, k, pos = torch.randn(64, 512, device="cuda").bfloat16(), torch.randn(64, 128, device="cuda").bfloat16(), i32(np.arange(64))
    return lambda **kw: op.run(q, k, pos, **kw)


def cache_read():
    p = Paged("bf16", "i8", 2, 64, 16, [300])
    return lambda **kw: p.cache.read(p.table, i32([0]), 300, **kw)


def attention_run():
    import torch
    p = Paged("bf16", "same", 2, 64, 16, [300])
    op = Attention("bf16", 8, 2, 64, page=16, max_tokens=100)
    q, past = torch.randn(100, 512, device="cuda").bfloat16(), i32([200])
    return lambda **kw: (op.run(q, p.cache, p.table, past, **kw),)


def attention_step():
    import torch
    p = Paged("bf16", "same", 2, 64, 16, [300] * 4)
    op = Attention("bf16", 8, 2, 64, page=16, max_seqs=4)
    q, past = torch.randn(4, 512, device="cuda").bfloat16(), i32([299, 5, 77, 150])
    return lambda **kw: (op.step(q, p.cache, p.table, past, **kw),)


@pytest.mark.parametrize("make", [head_norm, cache_read, attention_run, attention_step])
@pytest.mark.parametrize("pointer", [False, True])
def test_outputs_on_another_stream(make, pointer):
    # they do not lie in memory that work queued on the current stream still uses
    import torch
    run = make()
    want = run()
    big = torch.empty(1 << 28, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(stream=s)
    torch.cuda.synchronize()
    blocks = [torch.empty_like(t) for t in want for _ in range(8)]
    for _ in range(20):
        big.zero_()
    for b in blocks:
        b.fill_(7)
    used = {b.data_ptr() for b in blocks}
    del b, blocks
    got = run(stream=s.cuda_stream if pointer else s)
    assert not used & {t.data_ptr() for t in got}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("store", ["same", "i8"])
def test_captured_calls(store):
    # all operators in one graph, replayed with other inputs and positions, against eager calls
    import torch
    n, kv, dim = 3, 2, 64
    p = Paged("bf16", store, kv, dim, 16, [400, 40, 90])
    q = Paged("bf16", store, kv, dim, 16, [400, 40, 90])
    norm, op = HeadNorm("bf16", 8, kv, dim), Attention("bf16", 8, kv, dim, page=16, store=store, max_seqs=n, max_tokens=30)
    rows = torch.randn(30, (8 + 2 * kv) * dim, device="cuda").bfloat16()
    past, offsets = i32([300, 0, 17]), i32([0, 3, 20, 30])
    pos = i32(np.arange(30))

    def call(c):
        x = rows.clone()
        a, b = norm.run(x[:, :512], x[:, 512:640], pos)
        c.cache.write(b, x[:, 640:], c.table, past, offsets=offsets)
        y = op.run(a, c.cache, c.table, past, offsets=offsets)
        z = op.step(a[:n], c.cache, c.table, past)
        return (y, z, *c.cache.read(c.table, past, 30, offsets=offsets))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(p)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = call(p)
    for i in range(5):
        rows.copy_(torch.randn_like(rows.float()))
        past.copy_(i32([300 - 50 * i, 10 * (i % 2), 17 + i]))
        pos.add_(1000 * i)
        graph.replay()
        got = [t.clone() for t in outs]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, call(q)))


@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("f16", "same"), ("f32", "same"), ("bf16", "i8"), ("f16", "i8")])
@pytest.mark.parametrize("dim", [40, 64, 128, 200, 256])
def test_tiles_in_parts(dtype, store, dim):
    # from two parts of a tile to as many as there are, with sequences without rows, a last tile that is
    # not full, and windows that leave most parts empty
    for lens, past in (([3, 0, 17, 1], [500, 9, 512, 0]), ([40, 2], [1100, 3]), ([5], [6000])):
        for window in (0, 70):
            run_case(dtype, store, 12, 4, dim, 32, lens, past, window=window)


@pytest.mark.parametrize("past", [250, 1900])
def test_captured_parts(past):
    # replays with other pasts, between eager calls of the same handle
    import torch
    n, kv, dim = 2, 2, 64
    p = Paged("bf16", "same", kv, dim, 16, [past + 40, past + 40])
    op = Attention("bf16", 8, kv, dim, page=16, store="same", max_seqs=n, max_tokens=40)
    q = torch.randn(40, 8 * dim, device="cuda").bfloat16()
    at, offsets = i32([past, 3]), i32([0, 23, 40])
    rows = [torch.randn(2 * past, kv * dim, device="cuda").bfloat16() for _ in range(2)]
    p.cache.write(*rows, p.table, i32([0, 0]), offsets=i32([0, past, 2 * past]))
    run = lambda: op.run(q, p.cache, p.table, at, offsets=offsets)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = run()
    for i in range(5):
        q.copy_(torch.randn_like(q.float()))
        at.copy_(i32([past - 40 * i, 200 * (i % 2)]))
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, run())


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_a_cache_without_pages_and_a_table_without_entries(store, window):
    import torch
    empty, some = KVCache("bf16", 2, 64, 0, page=16, store=store), KVCache("bf16", 2, 64, 3, page=16, store=store)
    op = Attention("bf16", 4, 2, 64, page=16, store=store, window=window, max_seqs=3, max_tokens=9)
    q = torch.randn(9, 256, device="cuda").bfloat16()
    table, none = torch.zeros(3, 200, dtype=torch.int32, device="cuda"), torch.zeros(3, 0, dtype=torch.int32, device="cuda")
    for cache, t in ((empty, table), (empty, none), (some, none)):
        for past in ([0, 5, 3000], [-1, -2 ** 31, 2 ** 31 - 1]):
            assert not op.step(q[:3], cache, t, i32(past)).any()
            assert not op.run(q, cache, t, i32(past)).any()
    # the ends of the counts, with a table that has pages
    past = i32([-2 ** 31, 2 ** 31 - 1, -7])
    if window:
        assert not op.step(q[:3], some, table, past).any() and not op.run(q, some, table, past).any()
    else:
        y = op.step(q[:3], some, table, past)
        assert not y[0].any() and not y[2].any()


def test_calls_of_one_cache_from_threads():
    # different sequences, each thread on a stream of its own
    import sys
    import threading
    import torch
    cache = KVCache("bf16", 1, 8, 64, page=16)
    rows = [torch.randn(n, 8, device="cuda").bfloat16() for n in (3, 5, 16, 40)]
    tables = [torch.arange(16 * i, 16 * i + w, dtype=torch.int32, device="cuda")[None] for i, w in enumerate((1, 2, 5, 16))]
    past = i32([0])
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(300):
                cache.write(rows[i], -rows[i], tables[i], past)
                k, v = cache.read(tables[i], past, rows[i].shape[0])
                if not (torch.equal(k, rows[i]) and torch.equal(v, -rows[i])):
                    wrong.append(i)

    before = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(before)
    assert not wrong


def test_a_new_cache_is_written_on_another_stream():
    import torch
    x, past = torch.randn(64, 64, device="cuda").bfloat16(), i32([0])
    table, side = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)  # the current stream is busy while the cache is made
    cache = KVCache("bf16", 1, 64, 1, page=64)
    cache.write(x, x, table, past, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(t, x) for t in cache.read(table, past, 64))


@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("f16", "same"), ("f32", "i8"), ("bf16", "i8"), ("f16", "i8")])
@pytest.mark.parametrize("dim", [72, 88, 96, 104])
def test_heads_between_64_and_128_elements(dtype, store, dim):
    for page in (16, 128):
        run_case(dtype, store, 6, 2, dim, page, [150, 0, 1, 64, 300], [0, 3, 200, 64, 31], seed=dim)
    run_case(dtype, store, 6, 2, dim, 32, [1, 1, 1], [0, 300, -1], step=True)


@pytest.mark.parametrize("seqs,rows", [(1, 1), (5, 1), (3, 33), (70, 43), (2, 300)])
def test_equal_lengths(seqs, rows):
    # without offsets, against the same with them
    import torch
    past = [(37 * b) % 400 - (b % 7 == 3) * 1000 for b in range(seqs)]
    past = [max(p, -1) for p in past]
    a = run_case("bf16", "same", 6, 2, 64, 32, [rows] * seqs, past, equal=True)
    b = run_case("bf16", "same", 6, 2, 64, 32, [rows] * seqs, past)
    assert np.array_equal(a, b)


def test_offsets_of_no_order():
    # more rows in all than the call has: some stay as they were, none outside is touched, and the handle goes on
    import torch
    r = np.random.default_rng(7)
    n, seqs = 200, 150
    p = Paged("bf16", "same", 2, 64, 16, [300])
    op = Attention("bf16", 4, 2, 64, page=16, max_seqs=seqs, max_tokens=n)
    table = p.table.expand(seqs, -1)
    q = torch.randn(n + 2, 256, device="cuda").bfloat16()
    kv = torch.randn(n, 128, device="cuda").bfloat16()
    spare = KVCache("bf16", 2, 64, p.cache.pages, page=16)
    want = op.run(q[:50], p.cache, p.table, i32([100]))
    for _ in range(3):
        offsets = i32(np.concatenate([r.integers(-20, n + 20, seqs), [2 ** 31 - 1]]))
        past = i32(r.integers(-5, 400, seqs))
        out = torch.full((n + 2, 256), 5.0, device="cuda").bfloat16()
        op.run(q[1:-1], p.cache, table, past, offsets=offsets, out=out[1:-1])
        spare.write(kv, kv, table, past, offsets=offsets)
        spare.read(table, past, n, offsets=offsets)
        assert (out[0] == 5).all() and (out[-1] == 5).all()
    assert torch.equal(op.run(q[:50], p.cache, p.table, i32([100])), want)


@pytest.mark.parametrize("dtype,store,dim", [("bf16", "same", 64), ("f16", "i8", 96), ("f32", "same", 256)])
def test_tables_wider_than_the_sequences(dtype, store, dim):
    # tiles use fewer parts than their launch has: from one to all, side by side
    r = np.random.default_rng(5)
    lens, past = [3, 40, 1, 9, 2], [0, 250, 700, 1500, -1]
    held = [max(0, p + n) for p, n in zip(past, lens)]
    p = Paged(dtype, store, 2, dim, 16, held)
    wide = p.table.new_full((5, 600), -1)
    wide[:, :p.table.shape[1]] = p.table
    q = device(rounded(r.standard_normal((sum(lens), 4 * dim)), dtype), dtype)
    op = Attention(dtype, 4, 2, dim, page=16, store=store, max_seqs=5, max_tokens=sum(lens))
    offsets = i32(np.concatenate([[0], np.cumsum(lens)]))
    got = host(op.run(q, p.cache, wide, i32(past), offsets=offsets))
    at = 0
    for b, (n, s) in enumerate(zip(lens, past)):
        rows, at = slice(at, at + n), at + n
        g = got[rows].reshape(n, 4, dim)
        if s < 0:
            assert not g.any()
            continue
        y, a, bound = attend(host(q)[rows].reshape(n, 4, dim), *p.rows(b), 2, s, 0, np.ones(s + n, bool), None)
        assert_attention(g, y, a, bound, dtype, f"sequence {b}")
