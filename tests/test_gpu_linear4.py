"""Linear4 on the GPU against the formula in 64 bits: batches from one row to
several tiles, odd and tiny widths, groups, zero points, strided and unaligned
rows, values near the types' ends, infinities."""

import numpy as np
import pytest

from paper_2110_06037_amd import Linear4, native as N, quantize4
from tests.seq_util import assert_close, device, host, rounded, strided

pytestmark = pytest.mark.gpu


def weights(r, rows, cols, group, zero):
    groups = -(-cols // group)
    code = r.integers(0, 16, (rows, cols + cols % 2)).astype(np.uint8)
    scale = r.uniform(0.25, 1.0, (rows, groups)).astype(np.float16)
    scale[r.random((rows, groups)) < 0.1] *= -1
    z = r.integers(0, 16, (rows, groups)).astype(np.uint8) if zero else None
    at = np.arange(cols) // group
    w = (code[:, :cols].astype(np.float64) - (8 if z is None else z[:, at])) * scale[:, at].astype(np.float64)
    return code[:, 0::2] | (code[:, 1::2] << 4), scale, z, w


# roundings per term: the product, the sum within a wide product and over
# groups, waves and splits (a random walk over at most 2^20 terms would exceed
# no fixed count; sums here are trees of runs of at most 64 terms: 64 + 16),
# the scale and the bias; a sum around a non-zero code offset is up to 32
# times the size of the terms it leaves (codes below 16, offset 128 + 15)
COUNT = {"f32": 96, "f16": 96, "bf16": 96 * 32}


def run_case(dtype, m, cols, rows, group=128, zero=False, act="none", extra=0, bias=True, seed=0, scale_x=1.0):
    r = np.random.default_rng(seed)
    q, scale, z, w = weights(r, rows, cols, group, zero)
    b = np.asarray(r.uniform(-1, 1, rows), np.float32) if bias else None
    x = rounded(r.standard_normal((m, cols)) * scale_x, dtype)
    op = Linear4(dtype, q, scale, zero=z, bias=b, cols=cols, group=group, act=act)
    dx = strided(x, dtype, extra) if extra else device(x, dtype)
    y = op.run(dx)
    again = op.run(dx)
    exact = x @ w.T + (0 if b is None else b.astype(np.float64))
    size = np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b))
    exact = exact if act == "none" else np.maximum(exact, 0) if act == "relu" else np.clip(exact, 0, 6)
    assert_close(y, exact, size, dtype, COUNT[dtype], f"{dtype} {m}x{cols}x{rows}")
    assert np.array_equal(host(y), host(again))
    op.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 256])
def test_types_groups_and_zero_points(dtype, zero, group):
    run_case(dtype, 3, 640, 80, group, zero)
    run_case(dtype, 70, 328, 144, group, zero)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m", [1, 2, 5, 6, 11, 15, 16, 17, 31, 33, 48, 64, 65, 100, 129, 300])
def test_batches(dtype, m):
    run_case(dtype, m, 256, 96, 128, False)
    run_case(dtype, m, 200, 50, 64, True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols,rows", [(1, 1), (2, 3), (7, 16), (8, 17), (31, 15), (32, 16), (33, 40), (127, 65), (128, 64),
                                       (129, 1), (1000, 129), (1023, 200), (2048, 1000), (4100, 33), (8192, 64)])
def test_shapes(dtype, cols, rows):
    for m in (1, 4, 20, 90):
        run_case(dtype, m, cols, rows, 64, True, "relu6")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("extra", [1, 4, 8])
def test_strided_rows(dtype, extra):
    for m in (2, 40, 130):
        run_case(dtype, m, 264, 72, 32, False, "relu", extra, bias=False)


@pytest.mark.parametrize("dtype,scale_x", [("f32", 1e30), ("f32", 1e-30), ("bf16", 1e30), ("bf16", 1e-30), ("f16", 1e-5)])
def test_values_far_from_one(dtype, scale_x):
    run_case(dtype, 3, 512, 64, 128, True, bias=False, scale_x=scale_x)
    run_case(dtype, 80, 512, 64, 128, True, bias=False, scale_x=scale_x)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m", [3, 40, 96])
def test_infinities_and_nan_stay_in_their_rows(dtype, m):
    # an infinite input times a weight of either sign is that infinity, times a
    # weight of zero NaN; other rows of the batch keep their values
    r = np.random.default_rng(3)
    q, scale, z, w = weights(r, 48, 256, 128, True)
    x = rounded(r.standard_normal((m, 256)), dtype)
    op = Linear4(dtype, q, scale, zero=z, cols=256, group=128)
    clean = host(op.run(device(x, dtype)))
    x[0, 130], x[2, 5] = np.inf, np.nan
    got = host(op.run(device(x, dtype)))
    assert np.array_equal(got[1], clean[1]) and np.array_equal(got[3:], clean[3:])
    assert np.isnan(got[2]).all()
    col = w[:, 130]
    assert np.isnan(got[0, col == 0]).all()
    assert (got[0, col > 0] == np.inf).all() and (got[0, col < 0] == -np.inf).all()


def test_quantised_weights_stand_for_the_matrix():
    r = np.random.default_rng(4)
    w = r.standard_normal((40, 300)).astype(np.float32)
    for zero in (False, True):
        q, scale, z = quantize4(w, 64, zero)
        op = Linear4("f32", q, scale, zero=z, cols=300, group=64)
        got = host(op.run(device(np.eye(300), "f32"))).T
        # half a step, and the largest value of a symmetric group may lie half a step past code 15
        step = scale[:, np.arange(300) // 64].astype(np.float64)
        assert (np.abs(got - w) <= step * 1.01).all() and np.mean(np.abs(got - w) <= step * 0.51) > 0.95


def test_no_rows_in_place_and_refusals():
    import torch
    r = np.random.default_rng(5)
    q, scale, _, _ = weights(r, 64, 64, 32, False)
    op = Linear4("bf16", q, scale, group=32)
    assert op.run(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")).shape == (0, 64)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        op.run(x[:, :32])
    with pytest.raises(TypeError):
        op.run(x.half())
    with pytest.raises(ValueError):
        op.run(x, out=torch.zeros(2, 32, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        op.run(x.cpu())


def test_another_stream_and_graph_replays():
    import torch
    r = np.random.default_rng(6)
    q, scale, z, _ = weights(r, 500, 512, 128, True)
    op = Linear4("bf16", q, scale, zero=z, group=128)
    for m in (1, 20, 100):
        x = torch.randn(m, 512, device="cuda").bfloat16()
        want = op.run(x)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = op.run(x, stream=s)
        s.synchronize()
        assert torch.equal(got, want)
        y = torch.empty_like(want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            op.run(x, out=y)
        for _ in range(3):
            x.copy_(torch.randn(m, 512, device="cuda"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(op.run(x), y)


@pytest.mark.parametrize("m,cols,group", [(20, 2048, 128), (70, 2048, 128), (70, 4096, 64), (70, 2040, 32), (70, 2048, 96),
                                          (70, 8192, 32)])
def test_sums_of_bf16_inputs_have_float32_precision(m, cols, group):
    # Inputs of one sign whose second half repeats the first, against weights
    # that are its negative: every exact result is 0, and what comes out is the
    # error of the sums, almost unrounded.
    #
    # A rounding of a partial sum v is at most 2^-24 |v|, 2^-24 |v| / sqrt(3) in
    # the root mean square, and the errors of different roundings add like
    # their squares.  Codes may be summed around an offset that leaves them
    # below 32 (exact in bf16 beside 4 bits of code): the sums of 512 inputs
    # reach 24 * 512 * 1.5 scales, with up to 8 roundings of that size and 16 for each
    # 128 of them at a quarter of it: sqrt(8 + 4 * 16 / 16) * 18432 / sqrt(3) =
    # 36900 for 512 inputs.  Their terms' sizes are 3.7 * 1.5 in the mean, 2870
    # for 512: 13 of 2^-24 of the sizes, and 2048 inputs, four times, halve
    # that ratio: 6.5.  A factor of 2.5 above it: 16.
    r = np.random.default_rng(cols + group)
    rows, half = 80, cols // 2
    d = r.integers(-7, 8, (rows, half))
    code = np.concatenate([8 + d, 8 - d], 1).astype(np.uint8)
    x = rounded(1 + r.random((m, half)), "bf16")
    x = np.concatenate([x, x], 1)
    scale = np.ones((rows, -(-cols // group)), np.float16)
    op = Linear4("bf16", code[:, 0::2] | (code[:, 1::2] << 4), scale, cols=cols, group=group)
    got = host(op.run(device(x, "bf16")))
    size = x @ np.abs(code.astype(np.float64) - 8).T
    assert np.linalg.norm(got) <= 16 * 2.0 ** -24 * np.linalg.norm(size)
    op.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_groups_wider_than_the_rows(dtype):
    # one scale and zero point per row, up to the largest group there is
    for group in (1024, 1 << 30, (1 << 31) - 32):
        run_case(dtype, 3, 300, 40, group, True)
        run_case(dtype, 40, 300, 40, group, True)


@pytest.mark.parametrize("m,cols,group", [(3, 2048, 128), (20, 2048, 64), (70, 2048, 128), (70, 4096, 64), (70, 2048, 32)])
def test_sums_of_bf16_inputs_of_many_magnitudes(m, cols, group):
    # the same weights and bound as above (its ratios of partial sums to terms
    # do not depend on the inputs' sizes), on inputs whose sums need more bits
    # than float32 has
    r = np.random.default_rng(cols + group)
    rows, half = 80, cols // 2
    d = r.integers(-7, 8, (rows, half))
    code = np.concatenate([8 + d, 8 - d], 1).astype(np.uint8)
    x = rounded(np.exp(r.standard_normal((m, half))), "bf16")
    x = np.concatenate([x, x], 1)
    op = Linear4("bf16", code[:, 0::2] | (code[:, 1::2] << 4), np.ones((rows, -(-cols // group)), np.float16), cols=cols,
                 group=group)
    got = host(op.run(device(x, "bf16")))
    size = x @ np.abs(code.astype(np.float64) - 8).T
    assert np.linalg.norm(got) <= 16 * 2.0 ** -24 * np.linalg.norm(size)
    op.close()
