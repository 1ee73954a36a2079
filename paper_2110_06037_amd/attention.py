"""Python face of the attention operators (sn_op handles of the C ABI): the
norms of queries and keys with the position rotation, the paged cache of keys
and values, and attention over it.

They are called as the sequence operators are (``sequence``): packed rows that
may be strided, on the current stream of the handle's device or on ``stream``.
Three int32 device tensors say where a call's rows belong:

``offsets`` [seqs + 1]
    the sequences' first rows; without it they share the rows evenly;
``past`` [seqs]
    positions of each sequence before the call's rows (row i of sequence b
    stands at position past[b] + i); negative: no sequence in this slot;
``table`` [seqs, width]
    the pages of each sequence: position p lies in page table[b, p // page].
    Positions beyond the width, or of an entry outside 0 .. pages - 1, have no
    place: they are not written, read as zeros and are attended by nobody.
"""

from __future__ import annotations

import ctypes
import threading

import numpy as np

from . import native as N
from .sequence import _f32, _fp, _int, _Op


class HeadNorm(_Op):
    """Norms of queries and keys for each head, with the position rotation in the same pass.

    Each head's ``head_dim`` elements become x / sqrt(mean(x^2) + eps) * weight
    (``norm=False``: stay as they are), then each pair (a, b) of the first
    ``rot`` of them (default: all) is turned by t = position * freqs[j]::

        a cos t - b sin t,  b cos t + a sin t

    The pairs are (j, j + rot / 2) for ``pairs="halves"``, (2j, 2j + 1) for
    "neighbours"; ``freqs`` (float64 [rot / 2], radians) default to
    base ** (-2j / rot).  ``rot=0`` leaves the rotation out."""

    def __init__(self, dtype, heads, kv_heads, head_dim, q_weight=None, k_weight=None, norm=True, eps=1e-5, rot=None,
                 base=10000.0, freqs=None, pairs="halves", device=0):
        super().__init__(dtype, device)
        self.heads, self.kv_heads, self.head_dim = (
            _int(v, n, 0) for v, n in ((heads, "heads"), (kv_heads, "kv_heads"), (head_dim, "head_dim")))
        self.rot = rot = head_dim - head_dim % 2 if rot is None else _int(rot, "rot", 0)
        if freqs is None:
            freqs = float(base) ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
        freqs = np.ascontiguousarray(freqs, dtype=np.float64)
        if freqs.shape != (rot // 2,):
            raise ValueError(f"freqs has shape {freqs.shape}, not {(rot // 2,)}")
        qw, kw = _f32(q_weight, (head_dim,), "q_weight"), _f32(k_weight, (head_dim,), "k_weight")
        d = N.HeadNormDesc(self.dtype, heads, kv_heads, head_dim, rot, N.PAIRS[pairs], int(bool(norm)), eps)
        p = ctypes.c_void_p()
        N.check(self.lib.sn_headnorm_create(ctypes.byref(d), _fp(qw), _fp(kw), freqs.ctypes.data, device, ctypes.byref(p)))
        self._op, self._run = p, self.lib.sn_headnorm_run
        self._nq, self._nk = heads * head_dim, kv_heads * head_dim

    def run(self, q, k, positions=None, q_out=None, k_out=None, stream=None):
        """Enqueue on q [tokens, heads * head_dim], k [tokens, kv_heads * head_dim]
        (None where the handle has no such heads) and positions (int32 device
        tensor [tokens]); returns (q_out, k_out), which may be q and k."""
        if q is None and k is None:
            raise ValueError("neither q nor k is given")
        tokens, kind = (k if q is None else q).shape[0], self.torch_dtype
        side = None if stream is None else self._side(stream)
        qp = qs = kp = ks = qo = qos = ko = kos = 0
        if q is not None:
            nq = self._nq
            qp, qs = q.data_ptr(), self._rows(q, "q", tokens, nq, kind)
            if q_out is None:
                q_out, qos = q.new_empty((tokens, nq)) if side is None else self._new(q, (tokens, nq), kind, side), nq
            else:
                qos = self._rows(q_out, "q_out", tokens, nq, kind)
            qo = q_out.data_ptr()
        if k is not None:
            nk = self._nk
            kp, ks = k.data_ptr(), self._rows(k, "k", tokens, nk, kind)
            if k_out is None:
                k_out, kos = k.new_empty((tokens, nk)) if side is None else self._new(k, (tokens, nk), kind, side), nk
            else:
                kos = self._rows(k_out, "k_out", tokens, nk, kind)
            ko = k_out.data_ptr()
        pos = None if positions is None else _list(self, positions, "positions", tokens)
        st = self._current(self.device) if side is None else self._stream(side, (q, k, positions, q_out, k_out))
        rc = self._run(self._op, tokens, pos, qp, qs, kp, ks, qo, qos, ko, kos, st)
        if rc:
            N.check(rc)
        return q_out, k_out


def _list(op, t, name, n):
    """The address of an int32 device tensor of n values in one piece."""
    if t.dtype is op._torch.int32 and t.shape == (n,) and t.get_device() == op.device and (n <= 1 or t.stride(0) == 1):
        return t.data_ptr()
    raise ValueError(f"{name} is not a contiguous int32 tensor ({n},) on {op._dev}")


class _IO(threading.local):
    """The C argument of a thread's calls, filled anew by each."""

    def __init__(self):
        self.io = N.CacheIO()
        self.ref = ctypes.byref(self.io)


class _Paged(_Op):
    """What calls on a cache share: its geometry, and the C argument that names
    its memory and the call's sequences."""

    def __init__(self, dtype, kv_heads, head_dim, page, store, device):
        super().__init__(dtype, device)
        self.kv_heads, self.head_dim, self.page = (
            _int(v, n) for v, n in ((kv_heads, "kv_heads"), (head_dim, "head_dim"), (page, "page")))
        self.store = store
        self._desc = N.CacheDesc(self.dtype, N.STORE[store], kv_heads, head_dim, page)
        self._geometry = (self.dtype, store, kv_heads, head_dim, page, device)
        self._io = _IO()

    def _fill(self, cache, table, past, tokens, offsets):
        """The C argument of a call."""
        own, i32, device = self._io, self._torch.int32, self.device
        io = own.io
        seqs, width = table.shape
        if table.dtype is i32 and table.get_device() == device and (table.stride(1) == 1 or width <= 1):
            io.table_stride, io.table = table.stride(0) if seqs > 1 else width, table.data_ptr()
        else:
            raise ValueError(f"table is not an int32 tensor of contiguous rows on {self._dev}")
        io.past = _list(self, past, "past", seqs)
        io.offsets = None if offsets is None else _list(self, offsets, "offsets", seqs + 1)
        io.seqs, io.width, io.tokens = seqs, width, tokens
        io.pages, io.k, io.v, io.k_scale, io.v_scale = cache._memory
        return own.ref


class KVCache(_Paged):
    """A paged cache of keys and values: ``pages`` pages of ``page`` positions (a
    power of two from 16) of ``kv_heads`` heads of ``head_dim``.

    ``store="same"`` keeps rows in dtype; "i8" in 8 bits, each head's row x as the
    integers nearest to x / s with the scale s = max|x| * (1 / 127) in float32.  Its memory
    (``k``, ``v`` and with "i8" ``k_scale``, ``v_scale``) is in the operators' own
    order; rows come and go through ``write`` and ``read``."""

    def __init__(self, dtype, kv_heads, head_dim, pages, page=64, store="same", device=0):
        super().__init__(dtype, kv_heads, head_dim, page, store, device)
        self.pages = pages = _int(pages, "pages", 0)
        p = ctypes.c_void_p()
        N.check(self.lib.sn_cache_create(ctypes.byref(self._desc), device, ctypes.byref(p)))
        self._op = p
        self._tensors, self._memory = (None,) * 4, (pages, None, None, None, None)
        if device >= 0:
            torch, i8 = self._torch, store == "i8"

            def zeros(*shape, kind):
                return torch.zeros(pages, kv_heads, *shape, dtype=kind, device=self._dev)

            kind = torch.int8 if i8 else self.torch_dtype
            scales = [zeros(page, kind=torch.float32) if i8 else None for _ in range(2)]
            self._tensors = (zeros(page, head_dim, kind=kind), zeros(page // 16, head_dim, 16, kind=kind), *scales)
            self._memory = (pages, *(None if t is None else t.data_ptr() for t in self._tensors))
            torch.cuda.current_stream(device).synchronize()  # (a first write may come on another stream)

    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    k_scale = property(lambda self: self._tensors[2])
    v_scale = property(lambda self: self._tensors[3])

    def write(self, k, v, table, past, offsets=None, stream=None):
        """Enqueue the writing of the packed rows k, v [tokens, kv_heads * head_dim] to their places."""
        tokens, n = k.shape[0], self.kv_heads * self.head_dim
        ks, vs = self._rows(k, "k", tokens, n, self.torch_dtype), self._rows(v, "v", tokens, n, self.torch_dtype)
        io = self._fill(self, table, past, tokens, offsets)
        side = None if stream is None else self._side(stream)
        st = self._current(self.device) if side is None else self._stream(side, (k, v, table, past, offsets, *self._tensors))
        rc = self.lib.sn_cache_write(self._op, io, k.data_ptr(), ks, v.data_ptr(), vs, st)
        if rc:
            N.check(rc)

    def read(self, table, past, tokens, offsets=None, k_out=None, v_out=None, stream=None):
        """Enqueue the reading of the same places; returns (k, v) [tokens, kv_heads * head_dim]."""
        n, kind, at, outs = self.kv_heads * self.head_dim, self.torch_dtype, [], []
        io = self._fill(self, table, past, tokens, offsets)
        side = None if stream is None else self._side(stream)
        for out, name in ((k_out, "k_out"), (v_out, "v_out")):
            if out is None:
                out = past.new_empty((tokens, n), dtype=kind) if side is None else self._new(past, (tokens, n), kind, side)
                at += [out.data_ptr(), n]
            else:
                at += [out.data_ptr(), self._rows(out, name, tokens, n, kind)]
            outs.append(out)
        st = self._current(self.device) if side is None else self._stream(side, (*outs, table, past, offsets, *self._tensors))
        rc = self.lib.sn_cache_read(self._op, io, *at, st)
        if rc:
            N.check(rc)
        return outs[0], outs[1]


class Attention(_Paged):
    """Attention over a ``KVCache`` of the same geometry.

    Query head h of a row at position p sees the positions max(0, p - window + 1)
    .. p (``window=0``: 0 .. p) of key head h // (heads // kv_heads)::

        y = sum_j exp(scale * q k_j) v_j / sum_j exp(scale * q k_j)

    ``scale`` defaults to head_dim ** -0.5.  The rows' own keys and values are
    written to the cache before the call; a row that sees nothing is zeros.  The
    workspace holds calls of up to ``max_seqs`` sequences and ``max_tokens``
    rows in all (at least one a sequence); calls share it, so they must follow each other on one stream."""

    def __init__(self, dtype, heads, kv_heads, head_dim, page=64, store="same", scale=None, window=0, max_seqs=1,
                 max_tokens=1, device=0):
        super().__init__(dtype, kv_heads, head_dim, page, store, device)
        self.heads = heads = _int(heads, "heads")
        self.max_seqs, self.max_tokens = _int(max_seqs, "max_seqs"), _int(max_tokens, "max_tokens")
        self._n = heads * head_dim
        d = N.AttnDesc(self._desc, heads, _int(window, "window"), head_dim ** -0.5 if scale is None and head_dim > 0 else
                       float(scale or 0.0), max_seqs, max_tokens)
        p = ctypes.c_void_p()
        N.check(self.lib.sn_attn_create(ctypes.byref(d), device, ctypes.byref(p)))
        self._op = p

    def _call(self, f, q, cache, table, past, offsets, out, stream):
        if cache._geometry != self._geometry:
            raise ValueError(f"the cache is of (dtype, store, kv_heads, head_dim, page, device) {cache._geometry}, "
                             f"the handle of {self._geometry}")
        tokens, n, kind = q.shape[0], self._n, self.torch_dtype
        qs = self._rows(q, "q", tokens, n, kind)
        io = self._fill(cache, table, past, tokens, offsets)
        side = None if stream is None else self._side(stream)
        if out is None:
            out = q.new_empty((tokens, n)) if side is None else self._new(q, (tokens, n), kind, side)
            ys = n
        else:
            ys = self._rows(out, "out", tokens, n, kind)
        st = self._current(self.device) if side is None else self._stream(side, (q, out, table, past, offsets, *cache._tensors))
        rc = f(self._op, io, q.data_ptr(), qs, out.data_ptr(), ys, st)
        if rc:
            N.check(rc)
        return out

    def run(self, q, cache, table, past, offsets=None, out=None, stream=None):
        """Enqueue on the packed rows q [tokens, heads * head_dim]; returns y."""
        return self._call(self.lib.sn_attn_run, q, cache, table, past, offsets, out, stream)

    def step(self, q, cache, table, past, out=None, stream=None):
        """The same for one token of each of q.shape[0] sequences."""
        return self._call(self.lib.sn_attn_step, q, cache, table, past, None, out, stream)
