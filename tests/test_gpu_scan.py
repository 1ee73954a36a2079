"""Scan on the GPU against the recurrence in 64 bits, token by token: types,
head, group and state sizes, taps, lengths from none to many segments, packed
sequences, strided rows, carried and in-place windows and states, strong and
vanishing decays, values that are not finite, and the one-token kernel."""

import numpy as np
import pytest

from paper_2110_06037_amd import Scan, native as N
from tests.seq_util import assert_close, device, host, rounded, strided

pytestmark = pytest.mark.gpu

# Roundings per term, in units of 2^-24 of the size of what is summed: three
# convolved values of at most 5 + 5 (the sum of taps; exp2, reciprocal and
# products of silu) each, their products, the sums over state columns and
# tokens (trees of at most 64 + 8), the skip term.
COUNT = 128


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


class Case:
    """Weights, inputs and exact results of a set of sequences."""

    def __init__(self, dtype, lens, heads=4, dim=16, groups=1, state=16, conv=4, first=True, seed=0, step=(1e-3, 0.1),
                 rate=(1, 16), d=True, size=1.0):
        r = np.random.default_rng(seed)
        f32 = lambda v: np.asarray(v, np.float32)
        self.dtype, self.lens, self.first = dtype, lens, first
        self.heads, self.dim, self.groups, self.state, self.conv = heads, dim, groups, state, conv
        self.inner, self.seqs, self.tokens = heads * dim, len(lens), sum(lens)
        self.chans = self.inner + 2 * groups * state
        self.conv_w = f32(r.uniform(-1, 1, (self.chans, conv)) / np.sqrt(conv))
        self.conv_b = f32(r.uniform(-0.2, 0.2, self.chans))
        self.a = f32(-r.uniform(*rate, heads))
        self.d = f32(r.uniform(0.5, 1.5, heads)) if d else None
        s = np.exp(r.uniform(np.log(step[0]), np.log(step[1]), heads))
        self.dt_bias = f32(s + np.log(-np.expm1(-s)))
        self.x = rounded(r.standard_normal((self.tokens, self.chans)) * size, dtype)
        self.dt = rounded(r.standard_normal((self.tokens, heads)), dtype)
        self.window = rounded(r.standard_normal((self.seqs, conv - 1, self.chans)) * size, dtype) if first else None
        self.h0 = f32(r.standard_normal((self.seqs, heads, dim, state))).astype(np.float64) if first else None

    def op(self, **kw):
        kw = dict(dict(max_seqs=self.seqs, max_tokens=max(1, self.tokens)), **kw)
        return Scan(self.dtype, self.heads, self.dim, self.groups, self.state, self.conv_w, self.conv_b, self.a, self.d,
                    self.dt_bias, **kw)

    def offsets(self):
        import torch
        return torch.tensor(np.concatenate([[0], np.cumsum(self.lens)]), dtype=torch.int32, device="cuda")

    def carried(self):
        """(window, state) as device tensors, None where the case starts from zeros"""
        import torch
        if not self.first:
            return None, None
        return device(self.window, self.dtype), torch.from_numpy(self.h0.astype(np.float32)).cuda()

    def exact(self):
        """y, window, state and the sizes of y and state"""
        H, P, G, S, K = self.heads, self.dim, self.groups, self.state, self.conv
        w, b = self.conv_w.astype(np.float64), self.conv_b.astype(np.float64)
        a, bias = self.a.astype(np.float64), self.dt_bias.astype(np.float64)
        d = np.zeros(H) if self.d is None else self.d.astype(np.float64)
        y, ys = np.zeros((self.tokens, self.inner)), np.zeros((self.tokens, self.inner))
        wins, hs, hsizes = [], [], []
        row = 0
        for i, n in enumerate(self.lens):
            win = self.window[i] if self.first else np.zeros((K - 1, self.chans))
            h = self.h0[i].copy() if self.first else np.zeros((H, P, S))
            habs, size = np.abs(h), np.abs(h)
            for t in range(row, row + n):
                raw = np.concatenate([win, self.x[t:t + 1]])
                win = raw[1:]
                u = silu((raw.T * w).sum(1) + b)
                us = (np.abs(raw.T) * np.abs(w)).sum(1) + np.abs(b)
                X, Xs = u[:self.inner].reshape(H, P), us[:self.inner].reshape(H, P)
                B, Bs, C, Cs = (v.reshape(G, S).repeat(H // G, 0) for v in (
                    u[self.inner:self.inner + G * S], us[self.inner:self.inner + G * S],
                    u[self.inner + G * S:], us[self.inner + G * S:]))
                dt = np.logaddexp(0, self.dt[t] + bias)
                f = np.exp(dt * a)[:, None, None]
                # the decay's exponent is off by a few units of its own size
                # (the step size through two functions), each step by a few more
                grow = (0.05 + np.abs(dt * a) / 8)[:, None, None]
                size = f * (size + grow * habs) + (dt[:, None] * Xs)[..., None] * Bs[:, None]
                habs = f * habs + (dt[:, None] * Xs)[..., None] * Bs[:, None]
                h = f * h + (dt[:, None] * X)[..., None] * B[:, None]
                y[t] = ((h * C[:, None]).sum(-1) + d[:, None] * X).reshape(-1)
                ys[t] = ((size * Cs[:, None]).sum(-1) + np.abs(d)[:, None] * Xs).reshape(-1)
            row += n
            wins.append(win), hs.append(h), hsizes.append(size)
        return y, np.array(wins), np.array(hs), ys, np.array(hsizes)

    def check(self, got, exact=None):
        y, win, h, ys, hsize = exact or self.exact()
        assert_close(got[0], y, ys, self.dtype, COUNT, "y")
        assert np.array_equal(host(got[1]), win.reshape(got[1].shape)), "window"
        assert_close(got[2], h, hsize, "f32", COUNT, "state")

    def run(self, op, extra=0, **kw):
        win, h = self.carried()
        dev = (lambda v: strided(v, self.dtype, extra)) if extra else (lambda v: device(v, self.dtype))
        kw.setdefault("offsets", self.offsets())
        return op.run(dev(self.x), dev(self.dt), win, h, **kw)


def once(*args, extra=0, **kw):
    c = Case(*args, **kw)
    op = c.op()
    got = c.run(op, extra)
    c.check(got)
    again = c.run(op, extra)
    assert all(np.array_equal(host(a), host(b)) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("conv", [1, 2, 3, 4])
@pytest.mark.parametrize("first", [True, False])
def test_types_taps_and_starts(dtype, conv, first):
    once(dtype, [130, 3, 64], conv=conv, first=first, groups=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", [1, 3, 16, 31, 32, 33, 64, 72, 128, 130, 256])
def test_state_sizes(dtype, state):
    once(dtype, [70, 1], heads=2, dim=20, state=state)


@pytest.mark.parametrize("dim", [1, 3, 4, 15, 16, 33, 40, 63, 64, 65, 128, 130])
def test_head_sizes(dim):
    once("f16", [66, 5], heads=3, dim=dim, groups=3, state=24)


@pytest.mark.parametrize("heads,groups", [(1, 1), (5, 1), (6, 2), (9, 3), (8, 8), (24, 4)])
def test_heads_and_groups(heads, groups):
    once("bf16", [90, 33], heads=heads, groups=groups, state=16)


@pytest.mark.parametrize("lens", [[1], [2], [63], [64], [65], [127], [128], [129], [0, 1, 0, 64, 0], [0], [191, 1, 1, 320, 7],
                                  [1] * 70])
def test_lengths(lens):
    once("f32", lens, heads=2, state=16)
    once("bf16", lens, heads=2, state=16, first=False)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens", [[1000], [777, 0, 1300, 64]])
def test_long_sequences_in_segments(dtype, lens):
    once(dtype, lens, heads=4, dim=64, state=64)


@pytest.mark.parametrize("dtype,lens,conv", [("f16", [1, 79], 2), ("f32", [42, 2, 9, 28], 4), ("bf16", [157, 73], 3)])
def test_the_state_has_float32_precision_throughout(dtype, lens, conv):
    # A term's dozen roundings of at most 2^-24 each, uniform and independent,
    # have a root mean square of sqrt(12 / 3) = 2 of 2^-24, and a sum's errors
    # add like their squares: 4 of 2^-24 of the sizes in the mean over all
    # elements leaves a factor of 2 -- and shows a few terms of 11 bits among
    # many of 24, which the bound for single elements does not.
    c = Case(dtype, lens, heads=8, dim=64, state=128, conv=conv, first=False, seed=11)
    _, _, h, _, size = c.exact()
    err = host(c.run(c.op())[2]) - h
    assert np.linalg.norm(err) <= 4 * 2.0 ** -24 * np.linalg.norm(size)


@pytest.mark.parametrize("step,rate", [((1e-6, 1e-5), (1e-3, 1e-2)), ((0.5, 4), (4, 16)), ((20, 60), (16, 64)),
                                       ((1e-3, 0.1), (0, 0))])
def test_decays_from_none_to_vanishing(step, rate):
    # sums of hundreds of decades within a chunk, or a state that never decays
    once("f32", [200, 70], heads=6, step=step, rate=rate)
    once("f16", [200, 70], heads=6, step=step, rate=rate)


@pytest.mark.parametrize("dtype,size", [("f32", 1e6), ("bf16", 1e6), ("f32", 1e-6), ("bf16", 1e-6), ("f16", 1e-3)])
def test_values_far_from_one(dtype, size):
    # products of three values of 1e6 and far below one; nothing may pass through a narrower range
    c = Case(dtype, [150], heads=2, dim=32, state=32, size=size, seed=3)
    c.conv_b *= 0
    c.check(c.run(c.op()))


@pytest.mark.parametrize("extra", [1, 2, 8])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strided_and_unaligned_rows(extra, dtype):
    once(dtype, [100, 40], heads=4, dim=32, state=32, extra=extra)


def test_equal_lengths_without_offsets():
    c = Case("bf16", [75] * 3, heads=2)
    op = c.op()
    a = c.run(op)
    b = c.run(op, offsets=None)
    assert all(np.array_equal(host(u), host(v)) for u, v in zip(a, b))


def test_a_prompt_in_pieces_equals_it_in_one():
    # window and state carry a prompt over calls, in place
    whole = Case("f32", [300], heads=4, dim=32, state=32)
    win, h = whole.carried()
    op = whole.op()
    x, dt = device(whole.x, "f32"), device(whole.dt, "f32")
    parts = []
    for lo, hi in ((0, 1), (1, 3), (3, 100), (100, 100), (100, 228), (228, 300)):
        y, w2, h2 = op.run(x[lo:hi], dt[lo:hi], win, h, window_out=win, state_out=h, seqs=1)
        assert w2 is win and h2 is h
        parts.append(host(y))
    import torch
    whole.check((torch.from_numpy(np.concatenate(parts)), win, h))


@pytest.mark.parametrize("lens", [[2000], [700, 30, 0, 64]])
def test_in_place_equals_out_of_place(lens):
    c = Case("bf16", lens, heads=4, dim=64, state=64)
    op = c.op()
    want = c.run(op)
    win, h = c.carried()
    got = op.run(device(c.x, "bf16"), device(c.dt, "bf16"), win, h, window_out=win, state_out=h, offsets=c.offsets())
    assert all(np.array_equal(host(u), host(v)) for u, v in zip(want, got))


@pytest.mark.parametrize("lens", [[200], [1500]])
def test_values_that_are_not_finite_do_not_reach_back(lens):
    # in X, B, C and the step size: rows before keep their bits, other heads
    # and channels too, and rows after are NaN where the recurrence is not finite
    c = Case("bf16", lens, heads=4, dim=16, groups=2, state=16)
    op = c.op()
    clean = [host(v) for v in c.run(op)]
    bad = lens[0] - 90
    inner = c.inner
    for what, ch in (("x", 5), ("b", inner + 3), ("c", inner + 2 * 16 + 3), ("dt", 1)):
        for value in (np.nan, np.inf):
            x, dt = c.x.copy(), c.dt.copy()
            if what == "dt":
                dt[bad, ch] = value
            else:
                x[bad, ch] = value
            win, h = c.carried()
            y, w, hh = (host(v) for v in op.run(device(x, "bf16"), device(dt, "bf16"), win, h, offsets=c.offsets()))
            assert np.array_equal(y[:bad], clean[0][:bad]), (what, value)
            y4, c4, h4, hc = (v.reshape(-1, 4, 16) for v in (y, clean[0], hh.transpose(0, 3, 1, 2), clean[2].transpose(0, 3, 1, 2)))
            if what == "x":  # head 0, column 5; silu of an infinity of the tap's sign is 0 or infinite
                others = np.ones((4, 16), bool)
                others[0, 5] = False
                assert np.array_equal(y4[:, others], c4[:, others]) and np.array_equal(h4[:, others], hc[:, others])
                if np.isnan(value):
                    assert np.isnan(y4[bad:, 0, 5]).all() and np.isnan(h4[:, 0, 5]).all()
            elif what == "dt":
                keep = [0, 2, 3]
                assert np.array_equal(y4[:, keep], c4[:, keep]) and np.array_equal(h4[:, keep], hc[:, keep])
                assert not np.isfinite(y4[bad, 1]).any()
            else:  # group 0: heads 0 and 1
                assert np.array_equal(y4[:, 2:], c4[:, 2:])
                if np.isnan(value):
                    assert np.isnan(y4[bad, :2]).all()
                    if what == "c":  # read only: the state and rows past the taps keep their values
                        assert np.array_equal(hh, clean[2]) and np.array_equal(y[bad + 4:], clean[0][bad + 4:])


def test_sequences_do_not_touch():
    c = Case("f16", [70, 130, 20], heads=2)
    op = c.op()
    clean = [host(v) for v in c.run(op)]
    c.x[70:200] = np.nan
    c.window[1] = np.nan
    c.h0[1] = np.nan
    got = [host(v) for v in c.run(op)]
    assert np.array_equal(got[0][:70], clean[0][:70]) and np.array_equal(got[0][200:], clean[0][200:])
    assert np.array_equal(got[2][[0, 2]], clean[2][[0, 2]]) and np.isnan(got[0][70:200]).all()


def test_offsets_outside_the_rows_stay_inside():
    # offsets are device data that no host check sees: they are clamped
    import torch
    c = Case("bf16", [64, 64], heads=2)
    op = c.op()
    for bad in ([0, 500, 128], [-7, 64, 10 ** 9], [0, 128, 64], [0, 0, 0]):
        win, h = c.carried()
        y = torch.full((c.tokens, c.inner), 7.0, dtype=torch.bfloat16, device="cuda")
        op.run(device(c.x, "bf16"), device(c.dt, "bf16"), win, h, out=y,
               offsets=torch.tensor(bad, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
    got = c.run(op)
    c.check(got)


# ------------------------------------------------------------------ one token
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,dim,groups,state,conv", [(4, 64, 1, 128, 4), (6, 40, 3, 72, 3), (2, 1, 1, 1, 1), (3, 7, 1, 5, 2),
                                                         (2, 130, 2, 256, 4), (8, 64, 8, 16, 4), (1, 600, 1, 3, 4),
                                                         (5, 33, 5, 130, 4)])
def test_steps(dtype, heads, dim, groups, state, conv):
    for seqs in (1, 3, 33):
        for first in (True, False):
            c = Case(dtype, [1] * seqs, heads, dim, groups, state, conv, first)
            win, h = c.carried()
            op = c.op()
            exact = c.exact()
            c.check(op.step(device(c.x, dtype), device(c.dt, dtype), win, h), exact)
            if first:  # in place, twice from the same start
                for _ in range(2):
                    win, h = c.carried()
                    c.check(op.step(device(c.x, dtype), device(c.dt, dtype), win, h, window_out=win, state_out=h), exact)


def test_steps_follow_a_prompt():
    # a prompt, then tokens one by one, against the whole sequence at once
    import torch
    c = Case("bf16", [100], heads=4, dim=32, state=32)
    op = c.op()
    win, h = c.carried()
    x, dt = device(c.x, "bf16"), device(c.dt, "bf16")
    ys = [op.run(x[:80], dt[:80], win, h, window_out=win, state_out=h)[0]]
    for t in range(80, 100):
        ys.append(op.step(x[t:t + 1], dt[t:t + 1], win, h, window_out=win, state_out=h)[0])
    c.check((torch.cat(ys), win, h))


def test_steps_in_a_graph_and_on_another_stream():
    import torch
    c = Case("f16", [1] * 5, heads=4, dim=64, state=128)
    op = c.op()
    win, h = c.carried()
    x, dt = device(c.x, "f16"), device(c.dt, "f16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.check(op.step(x, dt, win, h, stream=s))
    s.synchronize()
    gw, gh, y = win.clone(), h.clone(), torch.empty(5, c.inner, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.step(x, dt, gw, gh, window_out=gw, state_out=gh, out=y)
    gw.copy_(win), gh.copy_(h)
    for _ in range(4):
        x.copy_(torch.randn_like(x))
        g.replay()
        torch.cuda.synchronize()
        ey, win, h = op.step(x, dt, win, h)
        assert torch.equal(ey, y) and torch.equal(win, gw) and torch.equal(h, gh)


def test_prompts_in_a_graph():
    import torch
    c = Case("bf16", [700, 64], heads=4, dim=64, state=64)
    op = c.op()
    want = c.run(op)
    win, h = c.carried()
    x, dt, off = device(c.x, "bf16"), device(c.dt, "bf16"), c.offsets()
    outs = [torch.empty_like(v) for v in want]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.run(x, dt, win, h, out=outs[0], window_out=outs[1], state_out=outs[2], offsets=off)
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_no_rows_and_refusals():
    import torch
    c = Case("bf16", [4], heads=2)
    op = c.op()
    win, h = c.carried()
    x, dt = device(c.x, "bf16"), device(c.dt, "bf16")
    y, w, s = op.run(x[:0], dt[:0], win, h)
    assert y.shape == (0, c.inner) and torch.equal(w, win) and torch.equal(s, h)
    y, w, s = op.run(x[:0], dt[:0])
    assert not w.any() and not s.any()
    with pytest.raises(ValueError):
        op.run(x[:, 1:], dt, win, h)
    with pytest.raises(ValueError):
        op.run(x, dt, win, h.half())
    with pytest.raises(ValueError):
        op.run(x, dt, win[:, :1], h)
    with pytest.raises(ValueError):
        op.run(x, dt, win, h, offsets=torch.tensor([0, 4], device="cuda"))
    for bad in (lambda: op.step(x, dt), lambda: op.run(x, dt, seqs=2)):
        with pytest.raises(N.SNError):  # more than max_seqs
            bad()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_stride_of_a_single_row_is_not_looked_at(dtype):
    import torch
    c = Case(dtype, [1], heads=2, first=True)
    op = c.op()
    for call, kw in ((op.step, {}), (op.run, {"seqs": 1})):
        f = op.lib.sn_scan_step if call == op.step else op.lib.sn_scan_run
        win, h = c.carried()
        x, dt = device(c.x, dtype), device(c.dt, dtype)
        y, w, s = call(x, dt, win, h, **kw)
        want = [t.clone() for t in (y, w, s)]
        for t in (y, w, s):
            t.fill_(7)
        io = op._io  # the same call again, with strides that say nothing
        io.x_stride = io.dt_stride = io.y_stride = 0
        N.check(f(op._op, io, torch.cuda.current_stream().cuda_stream))
        assert all(torch.equal(a, b) for a, b in zip(want, (y, w, s)))


@pytest.mark.parametrize("strong,dt", [(30, 200.0), (50, 120.0), (60, 1e4), (10, 1e4), (63, 50.0)])
def test_weak_decays_behind_strong_ones(strong, dt):
    # rows whose decay leaves nothing, then rows of a tenth and less in the same
    # chunk: the decays among the latter come from differences of the chunk's sums
    c = Case("f32", [64, 100], heads=4, dim=16, state=16, rate=(16, 16))
    c.dt[:strong] = dt
    c.dt[64:64 + strong] = dt
    c.dt_bias[:] = 0
    c.dt[strong:64] = -4.6
    c.dt[64 + strong:] = -4.6
    c.check(c.run(c.op()))


@pytest.mark.parametrize("dim", [16, 64])
@pytest.mark.parametrize("raw_dt", [-20.0, -30.0, -100.0])
@pytest.mark.parametrize("lens", [[1, 64, 40], [700]])
def test_states_held_by_vanishing_steps(lens, raw_dt, dim):
    # columns of zeros, no skip term, steps of almost nothing: y = C h alone,
    # beside products whose largest terms are 0 or far below one
    c = Case("f32", lens, heads=2, dim=dim, state=16, d=False, seed=5)
    c.conv_b[:] = 0
    c.dt_bias[:] = 0
    c.dt[:] = raw_dt
    c.x[:, :c.inner], c.window[:, :, :c.inner] = 0, 0
    exact = c.exact()
    op = c.op()
    c.check(c.run(op), exact)
    if lens[0] == 1:  # the same from the one-token kernel
        win, h = c.carried()
        y = op.step(device(c.x[:1], "f32"), device(c.dt[:1], "f32"), win[:1], h[:1])[0]
        assert_close(y, exact[0][:1], exact[3][:1], "f32", COUNT, "step")


@pytest.mark.parametrize("dim,state", [(16, 16), (64, 128)])
@pytest.mark.parametrize("rate", [(0.01, 0.05), (1, 16)])
@pytest.mark.parametrize("d", [True, False])
@pytest.mark.parametrize("bc,x,dt", [(300, 1, 0), (1000, 1, 50), (1000, 1000, 50), (1000, 1000, 1000)])
def test_rows_of_large_values_leave_the_others_their_precision(dim, state, rate, d, bc, x, dt):
    # within a chunk, in different rows: large B and C, X and steps, the rows
    # before and behind them as they always are
    c = Case("f32", [150], heads=2, dim=dim, state=state, rate=rate, d=d, seed=8)
    inner = c.inner
    c.x[52, inner:] *= bc
    c.x[110, inner:] *= bc
    c.x[47, :inner] *= x
    c.x[118, :inner] *= x
    if dt:
        c.dt[58] = dt
        c.dt[100] = dt
    c.check(c.run(c.op()))
