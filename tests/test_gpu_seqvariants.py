"""Variants of the sequence kernels that only larger calls take, against 64
bits: 4-bit products of several rows of blocks per workgroup (8192 features and
more) and of wide tiles (256 of them and more), scan steps of many quads per
thread, segments of more than two chunks, many segments at every width of the
state, and segments limited by the workspace; and of small calls, the batches of
every group size on both ways of loading, and the widest norms at any alignment."""

import pytest

from tests import test_gpu_blocknorm as norms
from tests.test_gpu_linear4 import run_case
from tests.test_gpu_scan import Case, once
from tests.seq_util import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [8200, 16390])
def test_products_of_many_features(dtype, group, rows):
    # 513 and 1025 rows of blocks: 2 or 4 to a workgroup, the last one cut; 264
    # inputs: 3 blocks of 128 in turns of two; 1 to 16 or 32 rows of x
    for m in (1, 3, 6, 16, 32):
        run_case(dtype, m, 264, rows, group, True, "relu")
    run_case(dtype, 5, 1160, rows, group, False, extra=8)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols,extra", [(264, 0), (259, 0), (392, 3)])
def test_products_of_many_tiles(dtype, group, cols, extra):
    # 18 tiles of rows of x by at least 17 of 256 features, both cut at the end,
    # with rows that allow wide loads and rows that do not
    run_case(dtype, 1100, cols, 4100, group, True, extra=extra)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,cols,group", [(33, 4200, 32), (70, 8328, 64), (40, 16520, 128)])
def test_products_of_many_runs(dtype, m, cols, group):
    run_case(dtype, m, cols, 80, group, True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("seqs,heads,dim,state", [(8, 64, 64, 128), (9, 64, 60, 128), (5, 64, 72, 128), (17, 32, 64, 100),
                                                  (3, 64, 200, 64), (2, 160, 64, 256)])
def test_steps_of_many_workgroups(dtype, seqs, heads, dim, state):
    c = Case(dtype, [1] * seqs, heads, dim, 2, state, 4)
    op, exact = c.op(), c.exact()
    x, dt = device(c.x, dtype), device(c.dt, dtype)
    win, h = c.carried()
    c.check(op.step(x, dt, win, h), exact)
    c.check(op.step(x, dt, win, h, window_out=win, state_out=h), exact)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", [33, 100, 128, 130, 256])
@pytest.mark.parametrize("dim", [40, 64])
def test_many_segments_at_every_width(dtype, state, dim):
    # per sequence: 6, 1, 2 and 3 segments of two chunks, from a given state
    once(dtype, [700, 100, 190, 300], heads=2, dim=dim, state=state)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens", [[1800], [1300, 0, 500]])
def test_segments_of_several_chunks(dtype, lens):
    # 29 chunks of 256 waves: 3 or 4 chunks to each of up to 10 segments
    once(dtype, lens, heads=64, dim=64, state=16, groups=4)


@pytest.mark.parametrize("lens", [[700] + [30] * 11, [70] * 12, [400] + [20] * 20])
def test_segments_limited_by_the_workspace(lens):
    # 4096 columns: states of 16 segments are held; 12 sequences leave room for
    # few beside their own, 21 for none
    once("bf16", lens, heads=64, dim=64, state=16)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", [264, 259])
def test_small_batches_of_every_group(dtype, group, cols):
    for m in (2, 6, 12, 20):
        run_case(dtype, m, cols, 90, group, True)


@pytest.mark.parametrize("dtype,res", [("f32", "f32"), ("f16", "f32"), ("f16", "f16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("dim", [600, 1500, 3001, 6002, 12001, 20001, 32767])
def test_norms_of_every_width_at_any_alignment(dtype, res, dim):
    norms.run_case(3, dim, dtype, res, "layer", "before", True, True, 1, "vector")
    norms.run_case(2, dim - dim % 8, dtype, res, "rms", "after", True, True, 1, 0.5, extra=1)
    norms.run_case(2, dim - dim % 8, dtype, res, "rms", "after", True, True, 1, 0.5)
