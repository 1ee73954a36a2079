"""A net's calls on several streams and from several threads on the GPU: its blocks share
workspaces, so each call's work waits for the last one's."""

import threading

import pytest

from paper_2110_06037_amd import SequenceNet
from tests.test_gpu_attnnet import ATTEND, SCAN
from workloads.sequence import sequence_weights

pytestmark = pytest.mark.gpu
SEQS = 2


@pytest.fixture
def net():
    with SequenceNet("bf16", sequence_weights([ATTEND, SCAN, ATTEND], seed=2), max_seqs=SEQS, max_tokens=600) as n:
        yield n


def rows(n, seed):
    import torch
    return torch.randn(n, 96, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def serial(net, prompt, tokens):
    state = net.new_state(SEQS, 400)
    return [net.run(prompt, state)] + [net.step(t, state) for t in tokens]


def test_a_call_waits_for_the_last_one_on_another_stream(net):
    import torch
    prompts, tokens = [rows(600, s) for s in (0, 1)], [[rows(SEQS, 10 * s + i) for i in range(3)] for s in (1, 2)]
    want = [serial(net, p, t) for p, t in zip(prompts, tokens)]
    states, streams = [net.new_state(SEQS, 400) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(4):
        for s, t, st, p, g in zip(streams, tokens, states, prompts, got):
            other = streams[1 - streams.index(s)]
            ended = torch.cuda.Event()
            with torch.cuda.stream(other):
                ended.record()
            with torch.cuda.stream(s):
                g.append(net.run(p, st) if i == 0 else net.step(t[i - 1], st))
                if s is streams[0]:
                    torch.cuda._sleep(20_000_000)
            s.synchronize()
            assert ended.query()  # (what the other stream had when the call was made)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_captured_steps_on_other_streams(net):
    import torch
    prompts, tokens = [rows(600, s) for s in (3, 4)], [[rows(SEQS, 10 * s + i) for i in range(6)] for s in (3, 4)]
    want = [serial(net, p, t) for p, t in zip(prompts, tokens)]
    states, streams = [net.new_state(SEQS, 400) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    for p, s in zip(prompts, states):
        net.run(p, s)
    graphs = [net.capture_step(s) for s in states]
    torch.cuda.synchronize()
    outs = [[], []]
    for i in range(6):
        for (token, out, replay), stream, t, o in zip(graphs, streams, tokens, outs):
            with torch.cuda.stream(stream):
                token.copy_(t[i])
                replay()
                o.append(out.clone())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o, w in zip(outs, want) for a, b in zip(o, w[1:]))


def test_threads(net):
    import torch
    n = 4
    prompts, tokens = [rows(600, s) for s in range(n)], [[rows(SEQS, 100 + 10 * s + i) for i in range(8)] for s in range(n)]
    want = [serial(net, p, t) for p, t in zip(prompts, tokens)]
    states, got = [net.new_state(SEQS, 400) for _ in range(n)], [None] * n
    torch.cuda.synchronize()

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            outs = [net.run(prompts[i], states[i])] + [net.step(t, states[i]) for t in tokens[i]]
            stream.synchronize()
        got[i] = outs

    threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_a_replay_waits_for_the_end_of_its_capture(net):
    # whose last work, the state's tensors as they were, is on the stream that was current
    import torch
    state, here = net.new_state(SEQS, 400), torch.cuda.Stream()
    net.run(rows(600, 7), state)
    torch.cuda.synchronize()
    with torch.cuda.stream(here):
        token, out, replay = net.capture_step(state)
        torch.cuda._sleep(20_000_000)
        ended = torch.cuda.Event()
        ended.record()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        replay()
    other.synchronize()
    assert ended.query()
