"""HeadNorm on the GPU against the formula in more than 64 bits: both kinds of
pairs, partial and no rotation, with and without norm and weights, head sizes
around the kernels' tiles, far and negative positions, strided and in-place rows."""

import numpy as np
import pytest

from paper_2110_06037_amd import HeadNorm, native as N
from tests.seq_util import assert_close, device, host, rounded, strided

pytestmark = pytest.mark.gpu
EPS = 1e-5


def angles(positions, freqs):
    """position * freq in [0, 2 pi), with the 64 bits of a long double's fraction."""
    ld = np.longdouble
    circle = 2 * ld("3.14159265358979323846264338327950288")
    turns = np.asarray(positions, ld)[:, None] * (np.asarray(freqs, ld) / circle)
    return (turns - np.floor(turns)) * circle


def formula(x, dim, w, positions, rot, freqs, pairs, norm):
    """(result, size of what each element is made from)"""
    h = x.reshape(x.shape[0], -1, dim)
    if norm:
        h = h / np.sqrt((h * h).mean(-1, keepdims=True) + EPS) * (1 if w is None else w)
    y, size = h.copy(), np.abs(h)
    if rot:
        t = angles(positions, freqs)[:, None]
        c, s = np.cos(t).astype(np.float64), np.sin(t).astype(np.float64)
        a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if pairs == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
        y[..., a], y[..., b] = h[..., a] * c - h[..., b] * s, h[..., b] * c + h[..., a] * s
        both = np.abs(h[..., a]) + np.abs(h[..., b])
        size[..., a], size[..., b] = both, both
    return y.reshape(x.shape), size.reshape(x.shape)


# roundings per term: the mean of up to 256 squares by a tree (12, halved by the
# root), its root (2), weights (2), sine and cosine (8), products and their sum (3)
COUNT = 24


def run_case(dtype, tokens, heads, kv, dim, rot=None, pairs="halves", norm=True, weights=True, positions=None, extra=0,
             base=10000.0, seed=0, in_place=False):
    import torch
    r = np.random.default_rng(seed)
    rot = dim - dim % 2 if rot is None else rot
    f32 = lambda v: np.asarray(v, np.float32).astype(np.float64)
    qw, kw = (f32(r.uniform(0.5, 1.5, dim)) for _ in range(2)) if norm and weights else (None, None)
    positions = r.integers(0, 100000, tokens) if positions is None else positions
    freqs = base ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    op = HeadNorm(dtype, heads, kv, dim, q_weight=qw, k_weight=kw, norm=norm, eps=EPS, rot=rot, base=base, pairs=pairs)
    q, k = (rounded(r.standard_normal((tokens, n * dim)) * 2, dtype) for n in (heads, kv))
    put = (lambda a: strided(a, dtype, extra)) if extra else (lambda a: device(a, dtype))
    dq, dk = put(q) if heads else None, put(k) if kv else None
    pos = torch.tensor(np.asarray(positions), dtype=torch.int32, device="cuda") if rot else None
    outs = op.run(dq, dk, pos, q_out=dq, k_out=dk) if in_place else op.run(dq, dk, pos)
    for got, x, w in zip(outs, (q, k), (qw, kw)):
        if got is None:
            assert x.shape[1] == 0
            continue
        y, size = formula(x, dim, w, positions, rot, freqs, pairs, norm)
        assert_close(got, y, size, dtype, COUNT, f"{tokens} x {dim}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("norm,weights", [(True, True), (True, False), (False, False)])
def test_every_form(dtype, pairs, norm, weights):
    for dim, rot in ((128, 128), (80, 40), (64, 0), (128, 64)):
        run_case(dtype, 5, 4, 2, dim, rot, pairs, norm, weights)


@pytest.mark.parametrize("dim,rot", [(1, 0), (2, 2), (3, 2), (7, 4), (8, 8), (16, 16), (31, 10), (40, 24), (63, 62), (64, 64),
                                     (65, 64), (72, 72), (96, 96), (127, 126), (128, 2), (129, 128), (136, 136), (192, 192),
                                     (200, 56), (255, 254), (256, 256), (256, 192)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_sizes(dim, rot, dtype):
    for pairs in ("halves", "neighbours"):
        run_case(dtype, 3, 3, 1, dim, rot, pairs)


@pytest.mark.parametrize("tokens", [1, 2, 63, 700])
@pytest.mark.parametrize("heads,kv", [(1, 0), (0, 1), (5, 5), (32, 8), (71, 1)])
def test_heads_and_tokens(tokens, heads, kv):
    run_case("bf16", tokens, heads, kv, 64)


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_far_and_negative_positions(pairs):
    far = [0, 1, -1, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31), 999999937, 123456789]
    for base in (10000.0, 1.0, 1e6):
        run_case("f32", len(far), 2, 1, 128, pairs=pairs, positions=far, base=base)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extra", [1, 4, 8, 13])
def test_strided_and_unaligned_rows(dtype, extra):
    for pairs in ("halves", "neighbours"):
        run_case(dtype, 9, 6, 2, 64, extra=extra, pairs=pairs)
        run_case(dtype, 9, 6, 2, 128, rot=96, extra=extra, pairs=pairs)


@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 96), (80, 80), (256, 256)])
def test_in_place(dim, rot):
    for pairs in ("halves", "neighbours"):
        run_case("bf16", 37, 5, 2, dim, rot, pairs, in_place=True)
        run_case("f16", 37, 5, 2, dim, rot, pairs, in_place=True, extra=3)


def test_own_frequencies_and_rows_that_are_not_finite():
    import torch
    freqs = np.array([3.0, -2.5, 100.0, 0.0])
    op = HeadNorm("f32", 2, 1, 8, freqs=freqs)
    r = np.random.default_rng(1)
    q, k = r.standard_normal((6, 16)).astype(np.float32), r.standard_normal((6, 8)).astype(np.float32)
    pos = np.array([0, 7, 1000, 5, 99999, 12])
    y, size = formula(q.astype(np.float64), 8, None, pos, 8, freqs, "halves", True)
    got = host(op.run(torch.from_numpy(q).cuda(), torch.from_numpy(k).cuda(), torch.tensor(pos, dtype=torch.int32).cuda())[0])
    assert_close(got, y, size, "f32", COUNT)
    bad = q.copy()
    bad[2, 3] = np.inf
    bad[4, 12] = np.nan
    again = host(op.run(torch.from_numpy(bad).cuda(), torch.from_numpy(k).cuda(), torch.tensor(pos, dtype=torch.int32).cuda())[0])
    touched = np.zeros_like(got, bool)
    touched[2, :8] = touched[4, 8:] = True
    assert np.array_equal(again[~touched], got[~touched]) and np.isnan(again[4, 8:]).all() and np.isnan(again[2, :8]).any()
    # zeros stay zeros, no rows are no work
    z = torch.zeros(2, 16, device="cuda")
    assert not op.run(z, z[:, :8].clone(), torch.zeros(2, dtype=torch.int32, device="cuda"))[0].any()
    assert op.run(z[:0], z[:0, :8], torch.zeros(0, dtype=torch.int32, device="cuda"))[0].shape == (0, 16)


def test_overlaps_are_refused_and_slices_taken():
    import torch
    op = HeadNorm("bf16", 4, 2, 64)
    wide = torch.randn(10, 64 * 8, device="cuda").bfloat16()
    q, k, pos = wide[:, :256], wide[:, 256:384], torch.arange(10, dtype=torch.int32, device="cuda")
    want = op.run(q, k, pos)
    for kw in (dict(q_out=wide[:, 64:320]), dict(k_out=wide[:, 320:448]), dict(q_out=wide[:, 256:512]), dict(k_out=wide[:, :128])):
        with pytest.raises(N.SNError) as e:
            op.run(q, k, pos, **kw)
        assert e.value.code == -1
    got = op.run(q, k, pos, q_out=q, k_out=wide[:, 384:])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
