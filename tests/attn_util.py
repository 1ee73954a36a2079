"""Helpers of the attention operators' tests: the operators in 64 bits, with the
bounds of a result's error, and caches with their lists on the device.

Bounds, derived before any run (u: the unit roundoff of the element type, 2^-8
bf16, 2^-11 f16, 2^-24 f32).  An attention output y = sum p v / sum p with
weights p = exp(scale q k) carries, with A = sum p |v| / sum p:

* one rounding of the result, u |y|;
* where the kernel rounds the weights and 8-bit values to the element type before
  their product (16-bit types), at most u A for each of the two, 2 u A;
* a score's error: q k is a float32 sum of dim products, off by at most
  (dim + 4) 2^-24 S with S = scale sum |q k| (its largest over the keys seen),
  which is the weight's relative error and enters numerator and denominator;
* float32 sums over n keys, n 2^-24 A in numerator and in denominator, and some
  roundings per weight (exp2, rescaling, reciprocal), 32.

So |got - y| <= u |y| + 2 u A (16-bit) + 2 A 2^-24 ((dim + 4) S + n + 32), and half
of the least step of f16 below 2^-14."""

import numpy as np

from tests.seq_util import FLOOR, UNIT, device, host, rounded, torch_type


def quantised(x, heads):
    """What rows [n, heads * dim] in 8 bits stand for."""
    h = x.reshape(x.shape[0], heads, -1)
    most = np.abs(h).max(-1)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        s = (most.astype(np.float32) * np.float32(1 / 127)).astype(np.float64)
        s = np.where(s < 2.0 ** -120, 0, s)
        code = np.where(s[..., None] > 0, np.rint(h / np.where(s > 0, s, 1)[..., None]), 0)
        out = code * s[..., None]
    return np.where(np.isfinite(h).all(-1)[..., None], out, np.nan).reshape(x.shape)


def attend(q, k, v, kv_heads, past, window, seen=None, scale=None):
    """(y, bound without the result's rounding) of rows q [n, heads, dim] over keys and
    values [past + n, kv_heads, dim]; `seen`: which positions have a place."""
    n, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    each = heads // kv_heads
    t = np.arange(k.shape[0])
    row = past + np.arange(n)[:, None]
    see = (t <= row) & (t > row - window if window else True)
    if seen is not None:
        see = see & seen
    y, a, s = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, heads, 1))
    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(heads):
            kk, vv = k[:, h // each], v[:, h // each]
            score = np.where(see, np.where(see, q[:, h] @ kk.T, 0) * scale, -np.inf)
            top = score.max(1, keepdims=True, initial=-np.inf)
            p = np.exp(np.where(see, score - np.where(np.isfinite(top), top, 0), -np.inf))
            total = p.sum(1, keepdims=True)
            p = p / np.where(total > 0, total, 1)
            # (values nobody sees take no part, whatever they are)
            if np.isfinite(vv).all():
                y[:, h], a[:, h] = p @ vv, p @ np.abs(vv)
            else:
                for i in range(n):
                    y[i, h], a[i, h] = p[i, see[i]] @ vv[see[i]], p[i, see[i]] @ np.abs(vv[see[i]])
            sizes = np.where(see, np.where(see, np.abs(q[:, h]) @ np.abs(kk).T, 0), 0)
            s[:, h, 0] = abs(scale) * sizes.max(1, initial=0)
    seen_keys = see.sum(1)[:, None, None]
    return y, a, 2 * a * 2.0 ** -24 * ((dim + 4) * s + seen_keys + 32)


def assert_attention(got, y, a, bound, dtype, what=""):
    fine = np.isfinite(y)
    assert got.shape == y.shape, (what, got.shape, y.shape)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: other values are finite"
    rough = 0 if dtype == "f32" else 2 * UNIT[dtype]
    limit = (UNIT[dtype] * np.abs(y) + (1 + UNIT[dtype]) * (rough * a + bound) + FLOOR[dtype])
    over = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, y, 0)) / np.where(fine, limit, 1), 0)
    assert over.size == 0 or over.max() <= 1, f"{what}: {over.max()} times the bound at {np.unravel_index(over.argmax(), over.shape)}"


class Paged:
    """A cache with its table on the device, full of NaN where nothing is written, and
    the same rows in 64 bits.  `held`: positions of each sequence."""

    def __init__(self, dtype, store, kv, dim, page, held, seed=0, spare=2, width=None, k=None, v=None):
        import torch
        from paper_2110_06037_amd import KVCache
        r = np.random.default_rng(seed)
        need = [-(-n // page) for n in held]
        self.pages = sum(need) + spare
        self.cache = KVCache(dtype, kv, dim, self.pages, page=page, store=store)
        poison(self.cache)
        order = r.permutation(self.pages)
        table = np.full((len(held), max([1, *need]) if width is None else width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = torch.from_numpy(table).cuda()
        n = sum(held)
        size_k, size_v = r.uniform(0.5, 1.5, kv * dim), r.uniform(0.2, 2, kv * dim)
        self.k = rounded(r.standard_normal((n, kv * dim)) * size_k, dtype) if k is None else k
        self.v = rounded(r.standard_normal((n, kv * dim)) * size_v, dtype) if v is None else v
        self.starts = np.concatenate([[0], np.cumsum(held)])
        if n:
            self.cache.write(device(self.k, dtype), device(self.v, dtype), self.table,
                             torch.zeros(len(held), dtype=torch.int32, device="cuda"),
                             offsets=torch.tensor(self.starts, dtype=torch.int32, device="cuda"))
        if store == "i8":
            self.k, self.v = quantised(self.k, kv), quantised(self.v, kv)
        self.k, self.v = (t.reshape(n, kv, dim) for t in (self.k, self.v))

    def rows(self, b):
        at = slice(self.starts[b], self.starts[b + 1])
        return self.k[at], self.v[at]


def poison(cache):
    """Every place as memory may be found: NaN, or codes with NaN for scales."""
    for t in (cache.k, cache.v):
        t.fill_(float("nan")) if t.is_floating_point() else t.fill_(-128)
    for t in (cache.k_scale, cache.v_scale):
        if t is not None:
            t.fill_(float("nan"))


def i32(values):
    import torch
    return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")
