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


def test_linear4_creation_refusals():
    from paper_2110_06037_amd import Linear4, quantize4
    q, scale, zero = quantize4(np.ones((4, 70)), 32, True)

    def make(q=q, scale=scale, zero=zero, cols=70, group=32, **kw):
        return Linear4("bf16", q, scale, zero=zero, cols=cols, group=group, device=kw.pop("device", -1), **kw)

    make().close()
    make(zero=None, bias=np.zeros(4), act="relu6").close()
    assert code(lambda: make(group=48, scale=scale[:, :2], zero=None)) == -2
    assert code(lambda: make(group=16, scale=np.ones((4, 5)), zero=None)) == -2
    bad = scale.copy()
    bad[1, 1] = np.inf
    assert code(lambda: make(scale=bad)) == -1
    assert code(lambda: make(zero=np.full_like(zero, 16))) == -1
    assert code(lambda: make(bias=np.full(4, np.nan))) == -1
    for wrong in (dict(cols=72), dict(scale=scale[:, :2]), dict(zero=zero[:3]), dict(bias=np.zeros(5))):
        with pytest.raises(ValueError):
            make(**wrong)
    L = N.lib()
    d = N.Linear4Desc(N.BF16, 0, 70, 32, 0)
    p = ctypes.c_void_p()
    assert L.sn_qlinear_create(ctypes.byref(d), q.ctypes.data, scale.ctypes.data, None, None, -1, ctypes.byref(p)) == -2
    d.rows, d.act = 4, 7
    assert L.sn_qlinear_create(ctypes.byref(d), q.ctypes.data, scale.ctypes.data, None, None, -1, ctypes.byref(p)) == -1
    d.act = 0
    assert L.sn_qlinear_create(ctypes.byref(d), None, scale.ctypes.data, None, None, -1, ctypes.byref(p)) == -1


def test_linear4_run_refusals_and_foreign_handles():
    from paper_2110_06037_amd import Linear4, quantize4
    L = N.lib()
    buf = np.zeros(256, np.uint16)
    p = buf.ctypes.data
    h = Linear4("bf16", *quantize4(np.ones((4, 8)), 32)[:2], cols=8, group=32, device=-1)
    norm = BlockNorm("bf16", 8, device=-1)

    def run(op=h._op, m=2, x=p, xs=8, y=p, ys=4):
        return L.sn_qlinear_run(op, m, x, xs, y, ys, None)

    assert run() == -5 and run(m=0, x=None, y=None) == -5
    assert run(m=-1) == -2 and run(m=262141) == -2
    assert run(x=None) == -1 and run(y=None) == -1 and run(x=p + 1) == -1
    assert run(xs=7) == -2 and run(ys=3) == -2
    assert run(op=norm._op) == -1 and run(op=None) == -1


def test_quantize4_rounds_to_the_nearest_code():
    from paper_2110_06037_amd import quantize4
    w = np.array([[7.5, -7.5, 0, 1, 2, 3, -1, 0.4]], np.float32)
    q, scale, zero = quantize4(w, 32)
    assert zero is None and scale.shape == (1, 1) and scale[0, 0] == 1
    codes = np.stack([q & 15, q >> 4], -1).reshape(1, -1)
    assert codes.tolist() == [[15, 0, 8, 9, 10, 11, 7, 8]]
    q, scale, zero = quantize4(np.array([[0.0, 15, 3, 7, 1]], np.float32), 32, True)
    assert scale[0, 0] == 1 and zero[0, 0] == 0
    assert np.stack([q & 15, q >> 4], -1).reshape(1, -1)[:, :5].tolist() == [[0, 15, 3, 7, 1]]


def _scan(**kw):
    from paper_2110_06037_amd import Scan
    o = dict(dtype="bf16", heads=4, head_dim=8, groups=2, state=16, conv_w=np.ones((4 * 8 + 2 * 2 * 16, 4)),
             a=-np.ones(4), max_seqs=3, max_tokens=100, device=-1)
    o.update(kw)
    return Scan(o.pop("dtype"), **o)


def test_scan_creation_refusals():
    _scan(d=np.ones(4), dt_bias=np.zeros(4), conv_b=np.zeros(96)).close()
    _scan(a=np.zeros(4)).close()
    w = np.ones((4 * 8 + 2 * 3 * 16, 4))
    assert code(lambda: _scan(groups=3, conv_w=w)) == -2
    assert code(lambda: _scan(conv_w=np.ones((96, 5)))) == -4
    assert code(lambda: _scan(heads=20000, head_dim=1, groups=20000, state=1, conv_w=np.ones((60000, 1)), a=np.zeros(20000))) == -4
    assert code(lambda: _scan(state=257, conv_w=np.ones((32 + 4 * 257, 4)))) == -4
    assert code(lambda: _scan(a=np.array([-1, -1, 0.5, -1]))) == -1
    assert code(lambda: _scan(a=np.array([-1, -1, -np.inf, -1]))) == -1
    assert code(lambda: _scan(dt_bias=np.full(4, np.nan))) == -1
    assert code(lambda: _scan(conv_w=np.full((96, 4), np.nan))) == -1
    assert code(lambda: _scan(max_seqs=0)) == -2 and code(lambda: _scan(max_seqs=65536)) == -2
    assert code(lambda: _scan(max_tokens=0)) == -2 and code(lambda: _scan(max_tokens=1 << 31)) == -2
    for wrong in (dict(conv_w=np.ones((95, 4))), dict(a=-np.ones(5)), dict(a=None), dict(d=np.ones(3))):
        with pytest.raises(ValueError):
            _scan(**wrong)


def test_scan_run_refusals():
    L = N.lib()
    handle = _scan()
    buf = np.zeros(1 << 16, np.uint8)
    p = buf.ctypes.data

    def call(step=False, op=handle._op, **kw):
        io = N.ScanIO()
        o = dict(seqs=2, tokens=2, x=p, x_stride=96, dt=p, dt_stride=4, window=p, state=p, y=p, y_stride=32, window_out=p,
                 state_out=p)
        o.update(kw)
        for k, v in o.items():
            setattr(io, k, v)
        return (L.sn_scan_step if step else L.sn_scan_run)(op, ctypes.byref(io), None)

    for step in (False, True):
        assert call(step) == -5
        assert call(step, seqs=-1) == -2 and call(step, seqs=4) == -2 and call(step, tokens=101) == -2
        assert call(step, x=None) == -1 and call(step, dt=None) == -1 and call(step, y=None) == -1
        assert call(step, x_stride=95) == -2 and call(step, y_stride=31) == -2 and call(step, dt_stride=3) == -2
        assert call(step, window=p + 1) == -1 and call(step, state=p + 2) == -1
        assert call(step, window_out=p + 64) == -1 and call(step, state_out=p + 64) == -1  # overlap, not in place
        assert call(step, window=None, state=None, window_out=None, state_out=None) == -5
        assert call(step, op=None) == -1
    assert call(tokens=3) == -2 and call(tokens=3, offsets=p) == -5
    assert call(seqs=0, tokens=1) == -2
    assert call(True, tokens=4) == -2 and call(True, offsets=p) == -2
    assert L.sn_scan_run(handle._op, None, None) == -1


def test_numbers_beyond_int32_are_refused():
    # they would arrive cut to 32 bits: a group of 2^32 + 32 as 32, with the
    # scales of one group per row
    from paper_2110_06037_amd import Linear4, quantize4
    q, scale, _ = quantize4(np.ones((4, 64)), 64)
    for group in ((1 << 32) + 32, 0, -32):
        with pytest.raises(ValueError):
            Linear4("bf16", q, scale, cols=64, group=group, device=-1)
    for wrong in (dict(max_seqs=(1 << 32) + 3), dict(device=(1 << 32) - 1)):
        with pytest.raises(ValueError):
            _scan(**wrong)
    with pytest.raises(ValueError):
        BlockNorm("bf16", 8, groups=(1 << 32) + 1, device=-1)
