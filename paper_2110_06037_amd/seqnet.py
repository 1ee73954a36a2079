"""A net of gated sequence blocks and attention blocks on the sequence and attention
operators, for inference.

Each block takes the normalised residual stream u and adds to the stream h; a
sequence block::

    z, raw, dt = split(in_proj(u))          # Linear4
    y = scan(raw, dt)                       # Scan: convolution, silu, state space scan
    v = norm(y * silu(z))                   # BlockNorm, in groups
    h = h + scale * out_proj(v)             # Linear4; the sum in the BlockNorm that
    u = norm(h)                             # also makes the next block's input

and an attention block::

    q, k, v = split(in_proj(u))             # Linear4
    q, k = turn(norm(q)), turn(norm(k))     # HeadNorm, in place
    cache.write(k, v)                       # KVCache
    y = attention(q, cache)                 # Attention
    h = h + scale * out_proj(y)             # as above
    u = norm(h)

A prompt of any length runs with ``run``, single tokens with ``step``; both
leave every block's convolution window and state, or its cache, behind in a
``SequenceState``.
"""

from __future__ import annotations

import threading

from .attention import Attention, HeadNorm, KVCache
from .sequence import BlockNorm, Linear4, Scan


class _Room:
    """Counts the positions that calls take of ``room`` for each sequence, and refuses calls
    that do not fit.

    The host keeps a bound of the largest count, as long as it knows of all that happened to
    ``past`` (another tensor, or another version of it, may hold anything).  Only where the bound
    does not do are the counts, and a call's offsets, read from the device."""

    def __init__(self, past, room):
        self.room, self._most, self._captured = room, 0, False
        self.know(past)

    def know(self, past):
        """``past`` holds what this has counted."""
        self._past, self._version = past, None if past.is_inference() else past._version

    def knows(self, past):
        return not self._captured and past is self._past and self._version is not None and past._version == self._version

    def take(self, past, seqs, rows, offsets=None, longest=None):
        if not rows:
            return
        if past.is_cuda:
            import torch
            if torch.cuda.is_current_stream_capturing():  # nobody tells how often that will run
                self._captured = True
                return
        if offsets is None:
            longest = -(-rows // seqs)
        most = self._most + (rows if longest is None else longest)
        if most > self.room or not self.knows(past):
            counts = past.tolist()
            if offsets is None:
                lens = [longest] * len(counts)
            else:
                at = offsets.tolist()
                lens = [b - a for a, b in zip(at, at[1:])]
            most = 0
            for b, (p, n) in enumerate(zip(counts, lens)):
                if p >= 0 and n > 0 and p + n > self.room:
                    raise ValueError(f"sequence {b} has {p} positions and gets {n} more, the state has room for {self.room}")
                most = max(most, p + max(n, 0) if p >= 0 else 0)
        self._most = most
        self.know(past)


class SequenceState:
    """What ``seqs`` sequences leave behind in every block (at first nothing).

    ``windows`` and ``states`` are the sequence blocks' (zeros: before the first
    token).  For attention blocks ``past`` (int32 [seqs]) counts the tokens so far (negative: no
    sequence in this slot; it may be set between calls), and ``caches`` hold ``room`` positions of each sequence:
    ``max_positions``, rounded up to the blocks' pages, in those that ``tables`` say.  A call
    that would take more is refused, before anything runs.  (Where the bound that the host keeps does not
    show that it fits, that reads ``past``, and waits for it.  In a graph that the caller captures, by other means than
    ``capture_step``, nothing is refused.)"""

    def __init__(self, net, seqs, max_positions=None):
        import torch
        dev = f"cuda:{net.device}"
        self.seqs = seqs
        scans = [b for b in net.blocks if not b.attends]
        attends = [b for b in net.blocks if b.attends]
        self.windows = [torch.zeros(seqs, b.scan.conv - 1, b.scan.chans, dtype=b.scan.torch_dtype, device=dev) for b in scans]
        self.states = [torch.zeros(seqs, b.scan.heads, b.scan.head_dim, b.scan.state, device=dev) for b in scans]
        self.past, self.caches, self.tables, self.room, self._room = None, [], [], None, None
        if attends:
            if max_positions is None:
                raise ValueError("a net with attention blocks needs max_positions")
            with torch.inference_mode(False):  # (a tensor with versions, wherever it is made)
                self.past = torch.zeros(seqs, dtype=torch.int32, device=dev)
            self.room = min(-(-max_positions // b.page) * b.page for b in attends)
            self._room = _Room(self.past, self.room)
        for b in attends:
            width = -(-max_positions // b.page)
            self.caches.append(b.new_cache(seqs * width))
            self.tables.append(torch.arange(seqs * width, dtype=torch.int32, device=dev).reshape(seqs, width))
        scan, cache = iter(zip(self.windows, self.states)), iter(zip(self.caches, self.tables))
        self.parts = [next(cache if b.attends else scan) for b in net.blocks]

    def tensors(self):
        """What a step reads and updates."""
        held = [t for c in self.caches for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]
        return self.windows + self.states + ([] if self.past is None else [self.past]) + self.tables + held


class _Block:
    attends = False

    def __init__(self, dtype, w, next_norm, max_seqs, max_tokens, device, eps):
        c = w["config"]
        inner, heads = c["heads"] * c["head_dim"], c["heads"]
        self.in_proj = Linear4(dtype, *w["in_proj"][:2], zero=w["in_proj"][2], cols=c["dim"], group=c["group"], device=device)
        self.scan = Scan(dtype, heads, c["head_dim"], c["groups"], c["state"], w["conv_w"], w["conv_b"], w["a"], w["d"],
                         w["dt_bias"], max_seqs=max_seqs, max_tokens=max_tokens, device=device)
        self.gate = BlockNorm(dtype, inner, post=w["gate_norm"], gate="before", groups=c["groups"], eps=eps, device=device)
        self.out_proj = Linear4(dtype, *w["out_proj"][:2], zero=w["out_proj"][2], cols=inner, group=c["group"], device=device)
        self.join = BlockNorm(dtype, c["dim"], pre=next_norm, scale=w["scale"], residual="f32", eps=eps, device=device)
        self.inner, self.chans = inner, self.scan.chans

    def close(self):
        for op in (self.in_proj, self.scan, self.gate, self.out_proj, self.join):
            op.close()

    def run(self, u, part, call):
        window, s = part
        p = self.in_proj.run(u)
        z, raw, dt = p[:, :self.inner], p[:, self.inner:self.inner + self.chans], p[:, self.inner + self.chans:]
        if call.step:
            y = self.scan.step(raw, dt, window, s, window_out=window, state_out=s)[0]
        else:
            y = self.scan.run(raw, dt, window, s, window_out=window, state_out=s, seqs=call.state.seqs, offsets=call.offsets)[0]
        self.gate.run(y, gate=z, out=y)
        return self.out_proj.run(y)


class _AttentionBlock:
    attends = True

    def __init__(self, dtype, w, next_norm, max_seqs, max_tokens, device, eps, shared):
        c = w["config"]
        heads, kv, dim = c["heads"], c["kv_heads"], c["head_dim"]
        self.page, self.nq, self.nk = c["page"], heads * dim, kv * dim
        self.in_proj = Linear4(dtype, *w["in_proj"][:2], zero=w["in_proj"][2], cols=c["dim"], group=c["group"], device=device)
        self.head_norm = HeadNorm(dtype, heads, kv, dim, w["q_norm"], w["k_norm"], eps=eps, rot=c["rot"], base=c["base"], device=device)
        # (it has no weights: one handle, and so one workspace, for all blocks that are alike)
        alike = (heads, kv, dim, c["page"], c["store"], c["window"])
        if alike not in shared:
            shared[alike] = Attention(dtype, heads, kv, dim, page=c["page"], store=c["store"], window=c["window"],
                                      max_seqs=max_seqs, max_tokens=max_tokens, device=device)
        self.attention = shared[alike]
        self.out_proj = Linear4(dtype, *w["out_proj"][:2], zero=w["out_proj"][2], cols=self.nq, group=c["group"], device=device)
        self.join = BlockNorm(dtype, c["dim"], pre=next_norm, scale=w["scale"], residual="f32", eps=eps, device=device)
        self.new_cache = lambda pages: KVCache(dtype, kv, dim, pages, page=c["page"], store=c["store"], device=device)

    def close(self):
        for op in (self.in_proj, self.head_norm, self.attention, self.out_proj, self.join):
            op.close()

    def run(self, u, part, call):
        cache, table = part
        p = self.in_proj.run(u)
        q, k, v = p[:, :self.nq], p[:, self.nq:self.nq + self.nk], p[:, self.nq + self.nk:]
        self.head_norm.run(q, k, call.positions if self.head_norm.rot else None, q_out=q, k_out=k)
        cache.write(k, v, table, call.state.past, offsets=call.offsets)
        if call.step:
            y = self.attention.step(q, cache, table, call.state.past)
        else:
            y = self.attention.run(q, cache, table, call.state.past, offsets=call.offsets)
        return self.out_proj.run(y)


class _Call:
    """What the blocks of one run or step share; ``positions`` of the rows where blocks attend."""

    def __init__(self, state, rows, offsets, step, longest=None, counted=True):
        self.state, self.offsets, self.step, self.counted = state, offsets, step, counted
        past = state.past
        if past is None:
            return
        if counted:
            state._room.take(past, state.seqs, rows, offsets, longest)
        import torch
        if step:
            self.lens, self.positions = 1, past
        elif offsets is None:
            self.lens = rows // state.seqs
            self.positions = (past[:, None] + torch.arange(self.lens, dtype=torch.int32, device=past.device)).reshape(-1)
        else:
            row = torch.arange(rows, dtype=torch.int32, device=past.device)
            seq = torch.searchsorted(offsets[1:], row, right=True).clamp_(max=state.seqs - 1)
            self.lens = offsets[1:] - offsets[:-1]
            self.positions = past[seq] + row - offsets[:-1][seq]

    def done(self):
        if self.state.past is not None:  # slots without a sequence stay so
            self.state.past += (self.state.past >= 0) * self.lens
            if self.counted:
                self.state._room.know(self.state.past)


class _Replay:
    """Replays a captured step.  The graph holds addresses only: this holds the
    net, whose handles own weights and workspaces, and the tensors."""

    def __init__(self, graph, net, state, *tensors):
        self.graph, self.net, self.state, self.tensors = graph, net, state, (state.tensors(), *tensors)
        self.past = state.past

    def __call__(self):
        with self.net._lock:
            if self.net.closed:
                raise RuntimeError("the net of this captured step is closed")
            self.net._turn()
            if self.past is not None:
                self.state._room.take(self.past, self.state.seqs, self.state.seqs)
            self.graph.replay()


class SequenceNet:
    """``weights``: {"norm": [dim] of the first block's input, "blocks": [...], each
    with its "config" (dim, heads, head_dim, groups, state, group), 4-bit
    "in_proj" and "out_proj" as ``quantize4`` gives them, "conv_w", "conv_b",
    "a", "d", "dt_bias", "gate_norm", the residual's "scale", and the "norm"
    [dim] that follows the block}.  An attention block's config has the "kind"
    "attention" (dim, heads, kv_heads, head_dim, rot, base, window, page, store,
    group), and beside the projections "q_norm" and "k_norm" [head_dim].  Inputs and outputs are [rows, dim] in
    ``dtype``; the residual stream between the blocks is float32.

    The blocks' handles have workspaces, one for all attention blocks that are alike, which every call uses.  So the net puts
    its calls (replays of captured steps among them) one after the other on the device, whatever streams and
    threads they come from; graphs that the caller captures by other means are the caller's to order."""

    def __init__(self, dtype, weights, max_seqs=1, max_tokens=1, device=0, eps=1e-5):
        blocks = weights["blocks"]
        self.device, self.closed = device, False
        self._lock, self._last = threading.RLock(), None  # the stream of the last call
        self.first = BlockNorm(dtype, blocks[0]["config"]["dim"], pre=weights["norm"], eps=eps, device=device)
        shared = {}
        self.blocks = [_AttentionBlock(dtype, w, w["norm"], max_seqs, max_tokens, device, eps, shared)
                       if w["config"].get("kind") == "attention" else
                       _Block(dtype, w, w["norm"], max_seqs, max_tokens, device, eps) for w in blocks]

    def close(self):
        with self._lock:
            self.closed = True
            self.first.close()
            for b in self.blocks:
                b.close()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def new_state(self, seqs=1, max_positions=None):
        """The state before the first token; attention blocks hold ``max_positions`` of each sequence."""
        return SequenceState(self, seqs, max_positions)

    def _turn(self):
        """A call's turn to queue its work, under the lock: behind the last call's, which may be on another stream."""
        import torch
        if torch.cuda.is_current_stream_capturing():
            return
        now = self.first._current(self.device)
        if now != self._last:
            if self._last is not None:
                torch.cuda.current_stream(self.device).wait_stream(torch.cuda.ExternalStream(self._last, device=self.first._dev))
            self._last = now

    def _forward(self, x, state, offsets, step, longest=None, counted=True):
        import torch
        with self._lock:
            self._turn()
            call = _Call(state, x.shape[0], offsets, step, longest, counted)
            u, _ = self.first.run(x)
            h = x.to(torch.float32, copy=True)  # updated below: never the caller's x
            for b, part in zip(self.blocks, state.parts):
                u, h = b.join.run(b.run(u, part, call), residual=h, res_out=h)
            call.done()
            return u

    def run(self, x, state, offsets=None, longest=None):
        """The normalised outputs [tokens, dim] of prompts in packed rows x
        (``offsets``: int32 device tensor of their first rows; none: of equal
        lengths), continuing from ``state``, which is brought up to date.
        ``longest``: how many rows the longest of them has, where the caller knows it (with
        ``offsets`` a call of more rows than the state has room for reads them otherwise)."""
        return self._forward(x, state, offsets, False, longest)

    def step(self, x, state):
        """The same for one token per sequence, x [seqs, dim]."""
        return self._forward(x, state, None, True)

    def capture_step(self, state):
        """A captured HIP graph of ``step`` on ``state``: (x, y, replay), where x
        is filled with the tokens before each replay() and y holds their outputs
        after it.  ``state`` is as before the capture; its tensors are what every
        replay updates.  ``replay`` keeps the net and them alive, and refuses to
        run once the net is closed, or where ``state`` has no room."""
        import torch
        with self._lock, torch.cuda.device(self.device):
            x = torch.zeros(state.seqs, self.first.dim, dtype=self.first.torch_dtype, device=f"cuda:{self.device}")
            # (what a step writes to a cache lies behind its sequence, until one that counts overwrites it)
            tensors = state.windows + state.states + ([] if state.past is None else [state.past])
            keep = [t.clone() for t in tensors]
            known = state.past is not None and state._room.knows(state.past)
            side = torch.cuda.Stream(self.device)
            side.wait_stream(torch.cuda.current_stream(self.device))
            with torch.cuda.stream(side):
                self._forward(x, state, None, True, counted=False)
            torch.cuda.current_stream(self.device).wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                y = self._forward(x, state, None, True, counted=False)
            self._turn()  # (the next call, on whatever stream, waits for the copies)
            for t, k in zip(tensors, keep):
                t.copy_(k)
            if known:
                state._room.know(state.past)
        return x, y, _Replay(graph, self, state, (x, y))
