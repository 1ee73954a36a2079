"""The sequence operators' handles without a device: argument checks of
creation and of runs (a host-only handle checks its arguments, then refuses)."""

import ctypes

import numpy as np
import pytest

from paper_2110_06037_amd import BlockNorm, native as N


def code(f):
    with pytest.raises(N.SNError) as e:
        f()
    return e.value.code


def test_norm_creation_refusals():
    one = np.ones(8)

    def make(dtype="bf16", dim=8, **kw):
        return BlockNorm(dtype, dim, device=kw.pop("device", -1), **kw)

    make(post=one).close()
    make(pre=one, residual="f32", scale=one).close()
    assert code(lambda: make(dim=0)) == -2
    assert code(lambda: make(dim=32769)) == -2
    assert code(lambda: make(groups=3)) == -2
    assert code(lambda: make(groups=0)) == -2
    assert code(lambda: make(groups=2, pre=one)) == -4
    assert code(lambda: make(eps=0.0)) == -1
    assert code(lambda: make(eps=float("nan"))) == -1
    assert code(lambda: make(scale=float("inf"))) == -1
    assert code(lambda: make(post_bias=one)) == -1
    assert code(lambda: make(residual="f16")) == -1
    assert code(lambda: make(device=-2)) == -1
    with pytest.raises(ValueError):
        make(post=np.ones(9))


def test_norm_run_refusals():
    L = N.lib()
    buf = np.zeros(64, np.float32)
    p = buf.ctypes.data
    handle = BlockNorm("f32", 8, pre=np.ones(8), residual="f32", device=-1)
    op = handle._op

    def run(rows=2, x=p, xs=8, g=0, gs=0, r=p, rs=8, ro=p, ros=8, y=p, ys=8):
        return L.sn_norm_run(op, rows, x, xs, g, gs, r, rs, ro, ros, y, ys, None)

    assert run() == -5 and run(rows=0) == -5          # sound, but no device
    assert run(rows=-1) == -2 and run(rows=1 << 62) == -2
    assert run(x=0) == -1 and run(r=0) == -1 and run(ro=0) == -1 and run(y=0) == -1
    assert run(xs=7) == -2 and run(ys=-8) == -2 and run(ros=9) == -2
    assert run(rows=1, xs=0, rs=0, ros=0, ys=0) == -5  # one row needs no stride
    assert run(g=p, gs=8) == -1                         # no gate in this handle
    assert run(x=p + 2) == -1                           # not on the elements' alignment
    assert L.sn_norm_run(None, 1, p, 8, 0, 0, p, 8, p, 8, p, 8, None) == -1
    assert L.sn_norm_create(None, None, None, None, None, None, -1, ctypes.byref(ctypes.c_void_p())) == -1
