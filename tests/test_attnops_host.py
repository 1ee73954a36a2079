"""The attention operators' handles without a device: argument checks of
creation and of runs (a host-only handle checks its arguments, then refuses)."""

import ctypes

import numpy as np
import pytest

from paper_2110_06037_amd import Attention, BlockNorm, HeadNorm, KVCache, native as N
from tests.attn_util import quantised


def code(f):
    with pytest.raises(N.SNError) as e:
        f()
    return e.value.code


def test_headnorm_creation_refusals():
    def make(dtype="bf16", heads=4, kv=2, dim=64, **kw):
        return HeadNorm(dtype, heads, kv, dim, device=kw.pop("device", -1), **kw)

    make().close()
    make(heads=0, q_weight=None, k_weight=np.ones(64)).close()
    make(dim=255, rot=100, pairs="neighbours", norm=False).close()
    assert code(lambda: make(heads=0, kv=0)) == -2 and code(lambda: make(heads=65536)) == -2
    assert code(lambda: make(dim=257)) == -2 and code(lambda: make(dim=0)) == -2
    assert code(lambda: make(rot=3, freqs=np.ones(1))) == -2 and code(lambda: make(rot=66, freqs=np.ones(33))) == -2
    assert code(lambda: make(eps=0.0)) == -1 and code(lambda: make(eps=float("inf"))) == -1
    assert code(lambda: make(norm=False, q_weight=np.ones(64))) == -1
    assert code(lambda: make(freqs=np.full(32, np.nan))) == -1 and code(lambda: make(freqs=np.full(32, 2.0 ** 20))) == -1
    assert code(lambda: make(device=-2)) == -1
    for wrong in (dict(q_weight=np.ones(63)), dict(freqs=np.ones(31)), dict(heads=(1 << 32) + 4), dict(dim=-1), dict(rot=-2)):
        with pytest.raises(ValueError):
            make(**wrong)
    with pytest.raises(KeyError):
        make(pairs="thirds")
    d = N.HeadNormDesc(N.BF16, 1, 1, 64, 64, 2, 1, 1e-5)
    p = ctypes.c_void_p()
    assert N.lib().sn_headnorm_create(ctypes.byref(d), None, None, np.ones(32).ctypes.data, -1, ctypes.byref(p)) == -1
    d.pairs, d.norm = 0, 2
    assert N.lib().sn_headnorm_create(ctypes.byref(d), None, None, np.ones(32).ctypes.data, -1, ctypes.byref(p)) == -1
    d.norm = 1
    assert N.lib().sn_headnorm_create(ctypes.byref(d), None, None, None, -1, ctypes.byref(p)) == -1


def test_headnorm_run_refusals():
    L = N.lib()
    buf = np.zeros(1024, np.float32)
    p = buf.ctypes.data
    op = HeadNorm("f32", 2, 1, 8, device=-1)
    still = HeadNorm("f32", 2, 0, 8, rot=0, device=-1)

    def run(h=op, tokens=2, pos=p, q=p, qs=16, k=p, ks=8, qo=p, qos=16, ko=p, kos=8):
        return L.sn_headnorm_run(h._op, tokens, pos, q, qs, k, ks, qo, qos, ko, kos, None)

    assert run() == -5 and run(tokens=0) == -5
    assert run(tokens=-1) == -2 and run(tokens=1 << 24) == -2
    assert run(q=None) == -1 and run(k=None) == -1 and run(qo=None) == -1 and run(ko=None) == -1 and run(pos=None) == -1
    assert run(qs=15) == -2 and run(ks=7) == -2 and run(qos=0) == -2 and run(kos=-8) == -2
    assert run(q=p + 2) == -1 and run(pos=p + 2) == -1
    assert run(qs=17) == -2                                    # in place with two strides
    assert run(tokens=1, qs=0, ks=0, qos=0, kos=0) == -5       # one row needs no stride
    assert run(still) == -1 and run(still, k=None, ko=None) == -1   # keys, positions it does not have
    assert run(still, k=None, ko=None, pos=None) == -5
    norm = BlockNorm("f32", 8, device=-1)
    assert run(norm) == -1 and L.sn_headnorm_run(None, 1, p, p, 8, p, 8, p, 8, p, 8, None) == -1


def test_cache_creation_refusals():
    def make(dtype="bf16", kv=2, dim=64, pages=4, **kw):
        return KVCache(dtype, kv, dim, pages, device=kw.pop("device", -1), **kw)

    make().close()
    make(store="i8", page=16).close()
    assert code(lambda: make(kv=0)) == -2 and code(lambda: make(kv=4097)) == -2
    assert code(lambda: make(dim=0)) == -2 and code(lambda: make(dim=12)) == -4 and code(lambda: make(dim=264)) == -4
    for page in (0, 8, 24, 8192, -16):
        assert code(lambda: make(page=page)) == -2
    assert code(lambda: make(kv=4096, dim=256, page=4096)) == -4     # a page of 2^33 bytes
    assert code(lambda: make(device=-2)) == -1
    for wrong in (dict(pages=-1), dict(pages=1 << 31), dict(dim=1 << 33)):
        with pytest.raises(ValueError):
            make(**wrong)
    with pytest.raises(KeyError):
        make(store="i3")
    d = N.CacheDesc(N.BF16, 2, 2, 64, 64)
    p = ctypes.c_void_p()
    assert N.lib().sn_cache_create(ctypes.byref(d), -1, ctypes.byref(p)) == -1
    assert N.lib().sn_cache_create(None, -1, ctypes.byref(p)) == -1


def test_attention_creation_refusals():
    def make(dtype="bf16", heads=4, kv=2, dim=64, **kw):
        return Attention(dtype, heads, kv, dim, device=kw.pop("device", -1), **kw)

    make().close()
    make(scale=0.0, window=5, store="i8", max_seqs=65535, max_tokens=1 << 20).close()
    assert code(lambda: make(heads=3)) == -2 and code(lambda: make(heads=0)) == -2 and code(lambda: make(heads=65536)) == -2
    assert code(lambda: make(dim=20)) == -4 and code(lambda: make(page=48)) == -2 and code(lambda: make(kv=0)) == -2
    assert code(lambda: make(window=-1)) == -2 and code(lambda: make(scale=float("nan"))) == -1
    assert code(lambda: make(max_seqs=0)) == -2 and code(lambda: make(max_seqs=65536)) == -2
    assert code(lambda: make(max_tokens=0)) == -2 and code(lambda: make(max_tokens=(1 << 26) + 1)) == -2
    with pytest.raises(ValueError):
        make(window=(1 << 32) + 5)


@pytest.mark.parametrize("store", ["same", "i8"])
def test_cache_and_attention_run_refusals(store):
    L = N.lib()
    buf = np.zeros(1 << 16, np.uint8)
    p = (buf.ctypes.data + 15) // 16 * 16
    s = p if store == "i8" else None
    cache = KVCache("bf16", 2, 64, 4, page=16, store=store, device=-1)
    attn = Attention("bf16", 4, 2, 64, page=16, store=store, max_seqs=3, max_tokens=100, device=-1)

    wide = KVCache("bf16", 64, 64, 4, page=64, store=store, device=-1)   # 2^42 rows in 2^30 pages
    wide_attn = Attention("bf16", 64, 64, 64, page=64, store=store, max_seqs=3, max_tokens=100, device=-1)

    def call(f, op=None, a=p, a_s=256, b=p, b_s=256, **kw):
        io = N.CacheIO()
        o = dict(pages=4, k=p, v=p, k_scale=s, v_scale=s, seqs=2, width=4, table=p, table_stride=4, past=p, tokens=2, offsets=None)
        o.update(kw)
        for k, v in o.items():
            setattr(io, k, v)
        h = op if op is not None else (cache if f in (L.sn_cache_write, L.sn_cache_read) else attn)
        return f(h._op, ctypes.byref(io), a, a_s, b, b_s, None)

    for f in (L.sn_cache_write, L.sn_cache_read, L.sn_attn_run, L.sn_attn_step):
        least = 128 if f in (L.sn_cache_write, L.sn_cache_read) else 256
        assert call(f) == -5 and call(f, seqs=0, tokens=0) == -5
        assert call(f, seqs=-1) == -2 and call(f, seqs=65536) == -2 and call(f, tokens=-1) == -2
        assert call(f, tokens=(1 << 26) + 1) == -2 and call(f, seqs=0) == -2
        assert call(f, pages=-1) == -2 and call(f, pages=1 << 31) == -2
        assert call(f, pages=1 << 30) == -5 and call(f, pages=1 << 30, op=wide if least == 128 else wide_attn, a_s=1 << 19, b_s=1 << 19) == -2
        assert call(f, width=-1) == -2 and call(f, width=(1 << 26) + 1) == -2
        assert call(f, k=None) == -1 and call(f, v=None) == -1 and call(f, k=p + 8) == -1 and call(f, v=p + 2) == -1
        assert call(f, pages=0, k=None, v=None) == -5
        assert call(f, table=None) == -1 and call(f, past=None) == -1 and call(f, table=p + 2) == -1 and call(f, past=p + 1) == -1
        assert call(f, table_stride=-1) == -2 and call(f, table_stride=0) == -5 and call(f, width=0, table=None) == -5
        assert call(f, a=None) == -1 and call(f, b=None) == -1 and call(f, a=p + 1) == -1
        assert call(f, a_s=least - 1) == -2 and call(f, b_s=least - 1) == -2
        if store == "i8":
            assert call(f, k_scale=None) == -1 and call(f, v_scale=p + 2) == -1
        else:
            assert call(f, k_scale=p) == -1
        assert f(cache._op if least == 128 else attn._op, None, p, 256, p, 256, None) == -1
        assert f(None, None, p, 256, p, 256, None) == -1
        assert call(f, op=attn if least == 128 else cache) == -1
    for f in (L.sn_attn_run, L.sn_attn_step):
        assert call(f, seqs=4, tokens=4) == -2
    assert call(L.sn_attn_run, tokens=102) == -2 and call(L.sn_attn_run, tokens=100) == -5
    for f in (L.sn_cache_write, L.sn_cache_read, L.sn_attn_run):
        assert call(f, tokens=3) == -2 and call(f, tokens=3, offsets=p) == -5 and call(f, tokens=3, offsets=p + 2) == -1
    many = Attention("bf16", 4, 2, 64, page=16, store=store, max_seqs=65535, device=-1)
    assert call(L.sn_attn_step, op=many, seqs=65535, tokens=65535, width=1 << 15, table_stride=0) == -4
    assert call(L.sn_attn_step, op=many, seqs=65535, tokens=65535, width=1 << 14, table_stride=0) == -5
    lots = Attention("bf16", 65535, 1, 64, page=16, store=store, max_tokens=1 << 20, device=-1)
    assert call(L.sn_attn_run, op=lots, seqs=1, tokens=(1 << 15) + 2, a_s=1 << 23, b_s=1 << 23) == -4
    assert call(L.sn_attn_step, tokens=4) == -2 and call(L.sn_attn_step, offsets=p) == -2


def test_a_cache_of_another_geometry_is_refused():
    import torch
    attn = Attention("bf16", 4, 2, 64, page=16, device=-1)
    q = torch.zeros(1, 256).bfloat16()
    table, past = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for kw in (dict(kv=1), dict(dim=128), dict(page=32), dict(store="i8"), dict(dtype="f16")):
        o = dict(dtype="bf16", kv=2, dim=64, page=16, store="same")
        o.update(kw)
        cache = KVCache(o["dtype"], o["kv"], o["dim"], 2, page=o["page"], store=o["store"], device=-1)
        with pytest.raises(ValueError):
            attn.step(q, cache, table, past)


def test_the_oracle_of_8_bit_rows():
    # codes by exact fractions, ties to even
    from fractions import Fraction
    r = np.random.default_rng(0)
    x = np.concatenate([r.standard_normal((20, 16)), r.integers(-127, 128, (20, 16)) / 2]).astype(np.float32).astype(np.float64)
    want = np.zeros_like(x)
    for i, row in enumerate(x):
        s = float(np.float32(np.abs(row).max()) * np.float32(1 / 127))
        want[i] = [round(Fraction(v) / Fraction(s)) * s if s else 0 for v in row]
    assert np.array_equal(quantised(x, 1), want)
