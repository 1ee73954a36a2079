"""Sequence operators on another stream than the current one: outputs that a
run makes itself do not lie in memory that work queued on the current stream
still uses."""

import numpy as np
import pytest

from paper_2110_06037_amd import BlockNorm, Linear4, Scan, quantize4

pytestmark = pytest.mark.gpu


def product():
    import torch
    r = np.random.default_rng(0)
    op = Linear4("bf16", *quantize4(r.standard_normal((512, 256)), 64)[:2], group=64)
    x = torch.randn(64, 256, device="cuda").bfloat16()
    return lambda **kw: (op.run(x, **kw),)


def scan():
    import torch
    r = np.random.default_rng(1)
    op = Scan("bf16", 8, 64, 1, 64, r.uniform(-1, 1, (640, 4)), a=-r.uniform(1, 16, 8), max_tokens=64)
    x, dt = torch.randn(64, 640, device="cuda").bfloat16(), torch.randn(64, 8, device="cuda").bfloat16()
    return lambda **kw: op.run(x, dt, **kw)


def norm():
    import torch
    op = BlockNorm("bf16", 512, pre=np.ones(512), residual="bf16")
    x, res = torch.randn(64, 512, device="cuda").bfloat16(), torch.randn(64, 512, device="cuda").bfloat16()
    return lambda **kw: op.run(x, residual=res, **kw)


@pytest.mark.parametrize("make", [product, scan, norm])
@pytest.mark.parametrize("pointer", [False, True])
def test_outputs_do_not_share_memory_with_queued_work(make, pointer):
    import torch
    run = make()
    want = run()
    big = torch.empty(1 << 28, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(stream=s)  # the side stream has its workspace, if any
    torch.cuda.synchronize()
    # blocks of the outputs' sizes whose last use waits behind some milliseconds of work
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


def test_the_current_stream_given_by_name_is_the_current_stream():
    import torch
    run = norm()
    want = run()
    for s in (torch.cuda.current_stream(), torch.cuda.current_stream().cuda_stream):
        assert all(torch.equal(a, b) for a, b in zip(want, run(stream=s)))
