"""The timed cases of the attention operators against their 64-bit form: what is
timed is also right, at the sizes that are timed."""

import pytest

from perf import more_operators as P
from tests.seq_util import UNIT

pytestmark = pytest.mark.gpu


def tensors(out):
    return list(out) if isinstance(out, (list, tuple)) else [out]


@pytest.mark.parametrize("name", [c["name"] for c in P.listed()])
def test_timed_cases(name, monkeypatch):
    # An output is one rounding (at most u of each value, so of the norm) of a
    # float32 result; the weights of 16-bit prompts are rounded once more, which moves
    # an output by at most u sum p |v| / sum p, and by u of the norm in the mean if the
    # roundings are independent.  float32 sums of up to 8192 products by trees and in order:
    # 2^-16 of the norm, as in the sequence operators' cases.
    import torch
    monkeypatch.setattr(P, "own", True)
    case = next(c for c in P.listed() if c["name"] == name)
    got, want = tensors(P.run(P.prepare(case, 7))), tensors(P.exact(case, 7))
    assert len(got) == len(want)
    for g, w in zip(got, want):
        assert g.shape == w.shape and bool(torch.isfinite(g).all())
        u = {torch.float32: UNIT["f32"], torch.float16: UNIT["f16"], torch.bfloat16: UNIT["bf16"]}[g.dtype]
        rounds = 2 if case["op"] == "attention" else 1
        # (8-bit rows of another scale's last bit take another code at some ties: half a step each)
        codes = 2.0 ** -9 if case.get("store") == "i8" and case["op"] == "cache" else 0
        assert float((g.double() - w).norm()) <= (rounds * u + codes + 2.0 ** -16) * float(w.norm())
