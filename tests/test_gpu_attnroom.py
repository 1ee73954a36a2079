"""A net's state on the GPU that has no room for a call's positions: prompts, steps
and replays are refused before anything runs, as long as it has them taken."""

import numpy as np
import pytest

from paper_2110_06037_amd import SequenceNet
from tests.attn_util import i32
from tests.test_gpu_attnnet import ATTEND, SCAN
from workloads.sequence import sequence_weights

pytestmark = pytest.mark.gpu


def rows(n):
    import torch
    return torch.randn(n, 96, device="cuda").bfloat16()


@pytest.fixture
def net():
    with SequenceNet("bf16", sequence_weights([ATTEND, SCAN, dict(ATTEND, page=32)], seed=1), max_seqs=3, max_tokens=128) as n:
        yield n


def refused(f, state):
    import torch
    before = [t.clone() for t in state.tensors()]
    with pytest.raises(ValueError, match="positions"):
        f()
    assert all(torch.equal(a, b) for a, b in zip(before, state.tensors()))


def test_steps_and_prompts_past_the_end(net):
    # 40 positions are 3 pages of 16 and 2 of 32: there is room for 48
    state = net.new_state(2, 40)
    refused(lambda: net.run(rows(98), state), state)
    net.run(rows(80), state)
    refused(lambda: net.run(rows(18), state), state)
    for _ in range(8):
        net.step(rows(2), state)
    assert state.past.tolist() == [48, 48]
    refused(lambda: net.step(rows(2), state), state)
    refused(lambda: net.run(rows(2), state), state)
    refused(lambda: net.run(rows(3), state, i32([0, 1, 3])), state)
    net.run(rows(0), state)


def test_packed_prompts_of_many_lengths(net):
    # what counts is each sequence's own end, not the rows of the call
    state = net.new_state(3, 48)
    net.run(rows(100), state, i32([0, 48, 52, 100]))
    assert state.past.tolist() == [48, 4, 48]
    refused(lambda: net.run(rows(1), state, i32([0, 0, 0, 1])), state)
    net.run(rows(44), state, i32([0, 0, 44, 44]))
    refused(lambda: net.run(rows(1), state, i32([0, 0, 1, 1])), state)


def test_replays(net):
    import torch
    state = net.new_state(2, 48)
    net.run(rows(92), state)
    token, out, replay = net.capture_step(state)
    replay(), replay()
    assert state.past.tolist() == [48, 48]
    refused(replay, state)
    # a state without room is captured as any other
    full = net.capture_step(state)[2]
    refused(full, state)
    state.past.copy_(i32([10, 0]))
    full(), replay()
    torch.cuda.synchronize()
    assert state.past.tolist() == [12, 2]


def test_counts_that_the_caller_sets(net):
    state = net.new_state(3, 48)
    net.run(rows(120), state)
    # a slot begins anew, another is empty
    state.past.copy_(i32([0, -1, 47]))
    net.step(rows(3), state)
    assert state.past.tolist() == [1, -1, 48]
    refused(lambda: net.step(rows(3), state), state)
    state.past[2] = -1
    for _ in range(47):
        net.step(rows(3), state)
    assert state.past.tolist() == [48, -1, -1]
    refused(lambda: net.step(rows(3), state), state)
    # more than was counted
    state.past.copy_(i32([0, 0, 0]))
    net.step(rows(3), state)
    state.past += 46
    net.step(rows(3), state)
    refused(lambda: net.step(rows(3), state), state)
    state.past = i32([40, 0, 0])
    refused(lambda: net.run(rows(27), state), state)
    net.run(rows(24), state)
    with __import__("torch").inference_mode():
        state = net.new_state(1, 48)
        net.run(rows(40), state)
        state.past += 7
        net.step(rows(1), state)
        refused(lambda: net.step(rows(1), state), state)


def test_a_net_without_attention_has_no_end():
    with SequenceNet("bf16", sequence_weights([SCAN], seed=1), max_seqs=1, max_tokens=128) as net:
        state = net.new_state(1)
        for _ in range(3):
            net.run(rows(128), state)
        net.step(rows(1), state)
