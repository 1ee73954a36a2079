"""BlockNorm on the GPU against the formula in 64 bits: every kind, gate, type
of residual, groups, widths around the kernels' tiles, odd widths, strided and
unaligned rows, in-place use, rows of zeros and of non-finite values."""

import numpy as np
import pytest

from paper_2110_06037_amd import BlockNorm, native as N
from tests.seq_util import assert_close, device, host, rounded, strided, torch_type

pytestmark = pytest.mark.gpu
EPS = 1e-5


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


def norm(t, kind, w, b, groups):
    """(normalised, bound of its error in units of 2^-24 given a relative error of 1 unit per input)"""
    v = t.reshape(t.shape[0], groups, -1)
    size = np.abs(v)
    if kind == "layer":
        mean = v.mean(-1, keepdims=True)
        size = size + np.abs(v).mean(-1, keepdims=True)
        v = v - mean
    k = 1 / np.sqrt((v * v).mean(-1, keepdims=True) + EPS)
    # an error of size * 2^-24 in v moves the mean square by at most 2 |v| size
    moved = np.abs(v) * k ** 3 * (np.abs(v) * size).mean(-1, keepdims=True)
    out, size = v * k, (size * k + moved + np.abs(v) * k)
    out, size = out.reshape(t.shape) * w, size.reshape(t.shape) * np.abs(w)
    return (out, size) if b is None else (out + b, size + np.abs(b))


def formula(x, gate, res, o):
    t, size = x, np.abs(x)
    if o["gate"] == "before":
        t, size = t * silu(gate), size * np.abs(silu(gate))
    if o["post"] is not None:
        t, size = norm(t, o["kind"], o["post"], o["post_bias"], o["groups"])
    if o["gate"] == "after":
        t, size = t * silu(gate), size * np.abs(silu(gate))
    s = 1.0 if o["scale"] is None else o["scale"]
    t, size = t * s, size * np.abs(s)
    r = None
    if res is not None:
        t, size = t + res, size + np.abs(res)
        r = (t, size)
    if o["pre"] is not None:
        # `size` is an absolute error scale: carry it through the second norm
        v = t - t.mean(-1, keepdims=True) if o["kind"] == "layer" else t
        k = 1 / np.sqrt((v * v).mean(-1, keepdims=True) + EPS)
        e = size + (size.mean(-1, keepdims=True) if o["kind"] == "layer" else 0)
        y = v * k * o["pre"] + (0 if o["pre_bias"] is None else o["pre_bias"])
        ys = (e * k + np.abs(v) * k ** 3 * (np.abs(v) * e).mean(-1, keepdims=True) + np.abs(v) * k) * np.abs(o["pre"])
        ys = ys + (0 if o["pre_bias"] is None else np.abs(o["pre_bias"]))
        return (y, ys), r
    return ((t, size) if r is None else None), r


# roundings per term: input conversions are exact; a gate (3), sums over a row by
# a tree (depth 6 + 8 elements + 16 waves), rsqrt (2), weights (2), scale, sum
COUNT = 24


def run_case(rows, dim, dtype, res=None, kind="rms", gate="none", post=True, pre=False, groups=1, scale=None, extra=0,
             seed=0, big=1.0):
    r = np.random.default_rng(seed)
    f32 = lambda v: np.asarray(v, np.float32).astype(np.float64)
    o = {"kind": kind, "gate": gate, "groups": groups,
         "post": f32(r.uniform(0.5, 1.5, dim)) if post else None,
         "post_bias": f32(r.uniform(-1, 1, dim)) if post and kind == "layer" else None,
         "pre": f32(r.uniform(0.5, 1.5, dim)) if pre else None,
         "pre_bias": f32(r.uniform(-1, 1, dim)) if pre and kind == "layer" else None,
         "scale": f32(r.uniform(0.1, 0.5, dim)) if scale == "vector" else scale if scale is None else f32(scale)}
    x = rounded(r.standard_normal((rows, dim)) * big, dtype)
    g = rounded(r.standard_normal((rows, dim)) * 2, dtype) if gate != "none" else None
    rs = rounded(r.standard_normal((rows, dim)) * 3, res) if res else None
    op = BlockNorm(dtype, dim, kind=kind, post=o["post"], post_bias=o["post_bias"], pre=o["pre"],
                   pre_bias=o["pre_bias"], scale=o["scale"], gate=gate, groups=groups, eps=EPS, residual=res)
    dev = (lambda a, t: strided(a, t, extra)) if extra else device
    y, ro = op.run(dev(x, dtype), gate=None if g is None else dev(g, dtype), residual=None if rs is None else dev(rs, res))
    ey, er = formula(x, g, rs, o)
    assert (y is None) == (ey is None) and (ro is None) == (er is None)
    if er is not None:
        assert_close(ro, er[0], er[1], res, COUNT, "res_out")
    if ey is not None:
        assert_close(y, ey[0], ey[1], dtype, COUNT, "y")
    op.close()


@pytest.mark.parametrize("dtype,res", [("f32", None), ("f32", "f32"), ("f16", None), ("f16", "f16"), ("f16", "f32"),
                                       ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "before", "after"])
def test_every_form(dtype, res, kind, gate):
    for post, pre in ((True, False), (True, True), (False, True)):
        for scale in (None, 0.22, "vector"):
            run_case(5, 192, dtype, res, kind, gate, post, pre, 1, scale)


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 63, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2056, 4095, 4096, 4097, 8192,
                                 8193, 16384, 16392, 32768])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_widths(dim, dtype):
    run_case(3, dim, dtype, "f32", "layer" if dim % 2 else "rms", "before", True, True, 1, "vector")


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 257])
@pytest.mark.parametrize("dim", [64, 520, 2048])
def test_rows(rows, dim):
    run_case(rows, dim, "bf16", "bf16", "rms", "after", True, True, 1, 0.5)


@pytest.mark.parametrize("dim,groups", [(64, 2), (96, 8), (4096, 8), (1001, 7), (24, 24), (8192, 2)])
@pytest.mark.parametrize("res", [None, "f32"])
def test_groups(dim, groups, res):
    run_case(6, dim, "f16", res, "rms", "before", True, False, groups, "vector" if res else None)


@pytest.mark.parametrize("extra", [1, 3, 8])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strided_and_unaligned_rows(extra, dtype):
    run_case(5, 256, dtype, dtype, "rms", "before", True, True, 1, 0.3, extra)


def test_in_place_and_another_stream():
    import torch
    r = np.random.default_rng(5)
    x, res = rounded(r.standard_normal((9, 640)), "bf16"), rounded(r.standard_normal((9, 640)), "bf16")
    op = BlockNorm("bf16", 640, pre=np.ones(640), scale=0.5, residual="bf16")
    a, b = op.run(device(x, "bf16"), residual=device(res, "bf16"))
    tx, tr = device(x, "bf16"), device(res, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c, d = op.run(tx, residual=tr, out=tx, res_out=tr, stream=s)
    s.synchronize()
    assert c is tx and d is tr
    assert np.array_equal(host(a), host(c)) and np.array_equal(host(b), host(d))


def test_rows_of_zeros_and_large_values():
    # a row of zeros normalises to the bias, by eps; 1e4 in f16 has a square
    # beyond f16's range, summed in float32
    op = BlockNorm("f16", 128, kind="layer", post=np.full(128, 2.0), post_bias=np.full(128, 0.25))
    y, _ = op.run(device(np.zeros((3, 128)), "f16"))
    assert np.array_equal(host(y), np.full((3, 128), 0.25))
    run_case(4, 256, "f16", None, "rms", big=1e4)
    run_case(4, 256, "f16", None, "layer", big=1e4)


def test_non_finite_rows_stay_alone():
    # infinities and NaN in one row, and gates at both ends: the other rows keep their values
    r = np.random.default_rng(1)
    x, g = rounded(r.standard_normal((6, 520)), "bf16"), rounded(r.standard_normal((6, 520)), "bf16")
    op = BlockNorm("bf16", 520, post=np.ones(520), gate="after")
    clean = host(op.run(device(x, "bf16"), gate=device(g, "bf16"))[0])
    x[1, 7], x[4, 519], g[2, 3], g[3, 0] = np.inf, np.nan, -200.0, 200.0
    got = host(op.run(device(x, "bf16"), gate=device(g, "bf16"))[0])
    keep = np.ones_like(got, bool)
    keep[1] = keep[4] = keep[2, 3] = keep[3, 0] = False
    assert np.array_equal(got[keep], clean[keep])
    assert np.isnan(got[4]).all() and np.isnan(got[1, 7]) and (got[1, np.arange(520) != 7] == 0).all()
    assert got[2, 3] == 0 and np.isfinite(got[3, 0])


def test_no_rows_and_refusals_on_the_device():
    import torch
    op = BlockNorm("bf16", 64, post=np.ones(64), residual="f32")
    y, r = op.run(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), residual=torch.empty(0, 64, device="cuda"))
    assert y is None and r.shape == (0, 64)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(N.SNError):
        op.run(x)  # the residual is missing
    with pytest.raises(TypeError):
        op.run(x.float(), residual=x.float())
    with pytest.raises(ValueError):
        op.run(x[:, :32], residual=x.float())
    with pytest.raises(ValueError):
        op.run(x, residual=torch.zeros(64, 2, device="cuda").t())
    with pytest.raises(ValueError):
        op.run(x, residual=torch.zeros(2, 64))


def test_graph_replays_equal_eager_runs():
    import torch
    op = BlockNorm("f16", 2048, pre=np.ones(2048), scale=0.5, residual="f32")
    x, r = torch.randn(3, 2048, device="cuda").half(), torch.randn(3, 2048, device="cuda")
    y, ro = torch.empty_like(x), torch.empty_like(r)
    op.run(x, residual=r, out=y, res_out=ro)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.run(x, residual=r, out=y, res_out=ro)
    for _ in range(3):
        x.copy_(torch.randn(3, 2048, device="cuda").half())
        g.replay()
        torch.cuda.synchronize()
        ey, er = op.run(x, residual=r)
        assert torch.equal(ey, y) and torch.equal(er, ro)


def test_more_rows_than_one_grid_dimension_has_threads_for():
    import torch
    op = BlockNorm("bf16", 8, post=np.arange(1, 9))
    rows = (1 << 26) + 5
    x = torch.empty(rows, 8, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(3))
    y = torch.zeros_like(x)
    op.run(x, out=y)
    for at in (0, (1 << 22) - 2, (1 << 25) + 7, (1 << 26) - 30, rows - 40):
        assert torch.equal(y[at:at + 40], op.run(x[at:at + 40])[0])
    assert bool((y != 0).any(dim=1).all())
