"""HeadNorm on the GPU: elements that do not rotate keep to themselves, infinities and NaN
included, whether a head's size comes in chunks or not."""

import numpy as np
import pytest

from paper_2110_06037_amd import HeadNorm
from tests.attn_util import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("dim,rot", [(7, 0), (7, 4), (65, 0), (65, 64), (65, 32), (72, 50), (129, 2), (200, 6), (255, 100),
                                     (64, 0), (64, 32), (80, 40), (128, 96), (72, 8)])
def test_what_is_not_finite_touches_its_own_pair_only(dtype, pairs, dim, rot):
    # row i has the bad value at element i; without the norm nothing else may change
    import torch
    op = HeadNorm(dtype, 2, 1, dim, norm=False, rot=rot, pairs=pairs)
    g = torch.Generator(device="cuda").manual_seed(dim)
    q, k = (torch.randn(dim, n * dim, generator=g, device="cuda").to(op.torch_dtype) for n in (2, 1))
    pos = i32(np.arange(dim) * 37) if rot else None
    clean = op.run(q, k, pos)
    at = torch.arange(dim, device="cuda")
    own = torch.zeros(dim, dim, dtype=torch.bool, device="cuda")  # [row][element that may change]
    own[at, at] = True
    turned = torch.arange(rot, device="cuda")
    own[turned, (turned + rot // 2) % max(rot, 1) if pairs == "halves" else turned ^ 1] = True
    for bad in (float("inf"), float("-inf"), float("nan")):
        bq, bk = q.clone(), k.clone()
        bq[at, dim + at], bk[at, at] = bad, bad
        for got, want, x, head in zip(op.run(bq, bk, pos), clean, (bq, bk), (1, 0)):
            got, want = got.view(dim, -1, dim), want.view(dim, -1, dim)
            assert torch.equal(got[:, head][~own], want[:, head][~own])
            assert head == 0 or torch.equal(got[:, 0], want[:, 0])
            # and what does not rotate is as it was
            assert torch.equal(torch.nan_to_num(got[:, :, rot:].float()), torch.nan_to_num(x.view(dim, -1, dim)[:, :, rot:].float()))
            assert not torch.isfinite(got[at, head, at]).any()
