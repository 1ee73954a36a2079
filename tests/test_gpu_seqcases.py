"""The timed cases of the sequence operators against their 64-bit form: what
is timed is also right, at the sizes that are timed."""

import pytest

from perf import operators as P
from tests.seq_util import UNIT

pytestmark = pytest.mark.gpu


def tensors(out):
    return list(out) if isinstance(out, (list, tuple)) else [out]


@pytest.mark.parametrize("name", [c["name"] for c in P.listed()])
def test_timed_cases(name, monkeypatch):
    # An output is one rounding (at most u of each value, so of the norm) of a
    # float32 result.  That is summed by a tree of some 80 roundings of partial
    # sums that are no larger, in the mean, than the sum: sqrt(80) 2^-24 < 2^-20
    # of the norm if the errors are independent; 2^-16 leaves a factor of 16.
    import torch
    monkeypatch.setattr(P, "own", True)
    case = next(c for c in P.listed() if c["name"] == name)
    got, want = tensors(P.run(P.prepare(case, 7))), tensors(P.exact(case, 7))
    assert len(got) == len(want)
    for g, w in zip(got, want):
        assert (g is None) == (w is None)
        if g is None:
            continue
        assert g.shape == w.shape and bool(torch.isfinite(g).all())
        u = {torch.float32: UNIT["f32"], torch.float16: UNIT["f16"], torch.bfloat16: UNIT["bf16"]}[g.dtype]
        assert float((g.double() - w).norm()) <= (u + 2.0 ** -16) * float(w.norm())
