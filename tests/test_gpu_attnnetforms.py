"""Attention blocks without a rotation in a net on the GPU, alone and beside others: prompts
and tokens against the same net in 64 bits, captured steps against eager ones."""

import numpy as np
import pytest

from paper_2110_06037_amd import SequenceNet
from tests.gpu_util import TOL
from tests.seq_util import device, host, rounded
from tests.test_gpu_attnnet import ATTEND, SCAN, exact
from tests.test_gpu_seqnet import off
from workloads.sequence import sequence_weights

pytestmark = pytest.mark.gpu
STILL = dict(ATTEND, rot=0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("blocks", [[STILL], [SCAN, STILL, ATTEND, dict(STILL, window=20)]])
def test_blocks_without_a_rotation(dtype, blocks):
    import torch
    weights = sequence_weights(blocks, seed=3)
    r = np.random.default_rng(4)
    xs = [rounded(r.standard_normal((n, 96)), dtype) for n in (40, 1, 33)]
    want = [exact(weights, x) for x in xs]
    with SequenceNet(dtype, weights, max_seqs=3, max_tokens=74) as net:
        offsets = torch.tensor([0, 40, 41, 74], dtype=torch.int32, device="cuda")
        got = host(net.run(device(np.concatenate(xs), dtype), net.new_state(3, 80), offsets))
        for g, w in zip(np.split(got, [40, 41]), want):
            assert off(g, w) <= TOL[dtype]
        state, x = net.new_state(1, 40), device(xs[0], dtype)
        parts = [net.run(x[:30], state)] + [net.step(x[t:t + 1], state) for t in range(30, 40)]
        assert off(host(torch.cat(parts)), want[0]) <= TOL[dtype]


def test_captured_steps_without_a_rotation():
    import torch
    with SequenceNet("bf16", sequence_weights([STILL, SCAN, ATTEND], seed=5), max_seqs=2, max_tokens=32) as net:
        eager, captured = net.new_state(2, 40), net.new_state(2, 40)
        x = torch.randn(32, 96, device="cuda").bfloat16()
        net.run(x, eager), net.run(x, captured)
        token, out, replay = net.capture_step(captured)
        for _ in range(4):
            t = torch.randn(2, 96, device="cuda").bfloat16()
            token.copy_(t)
            replay()
            want = net.step(t, eager)
            torch.cuda.synchronize()
            assert torch.equal(want, out)
