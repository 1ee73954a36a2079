"""A net of gated sequence blocks on the sequence operators, for inference.

Each block takes the normalised residual stream u and adds to the stream h::

    z, raw, dt = split(in_proj(u))          # Linear4
    y = scan(raw, dt)                       # Scan: convolution, silu, state space scan
    v = norm(y * silu(z))                   # BlockNorm, in groups
    h = h + scale * out_proj(v)             # Linear4; the sum in the BlockNorm that
    u = norm(h)                             # also makes the next block's input

A prompt of any length runs with ``run``, single tokens with ``step``; both
leave every block's convolution window and state behind in a ``SequenceState``.
"""

from __future__ import annotations

from .sequence import BlockNorm, Linear4, Scan


class SequenceState:
    """The windows and states of ``seqs`` sequences in every block (zeros: before the first token)."""

    def __init__(self, net, seqs):
        import torch
        dev = f"cuda:{net.device}"
        self.seqs = seqs
        self.windows = [torch.zeros(seqs, b.scan.conv - 1, b.scan.chans, dtype=b.scan.torch_dtype, device=dev)
                        for b in net.blocks]
        self.states = [torch.zeros(seqs, b.scan.heads, b.scan.head_dim, b.scan.state, device=dev) for b in net.blocks]


class _Block:
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


class _Replay:
    """Replays a captured step.  The graph holds addresses only: this holds the
    net, whose handles own weights and workspaces, and the tensors."""

    def __init__(self, graph, net, *tensors):
        self.graph, self.net, self.tensors = graph, net, tensors

    def __call__(self):
        if self.net.closed:
            raise RuntimeError("the net of this captured step is closed")
        self.graph.replay()


class SequenceNet:
    """``weights``: {"norm": [dim] of the first block's input, "blocks": [...], each
    with its "config" (dim, heads, head_dim, groups, state, group), 4-bit
    "in_proj" and "out_proj" as ``quantize4`` gives them, "conv_w", "conv_b",
    "a", "d", "dt_bias", "gate_norm", the residual's "scale", and the "norm"
    [dim] that follows the block}.  Inputs and outputs are [rows, dim] in
    ``dtype``; the residual stream between the blocks is float32."""

    def __init__(self, dtype, weights, max_seqs=1, max_tokens=1, device=0, eps=1e-5):
        blocks = weights["blocks"]
        self.device, self.closed = device, False
        self.first = BlockNorm(dtype, blocks[0]["config"]["dim"], pre=weights["norm"], eps=eps, device=device)
        self.blocks = [_Block(dtype, w, w["norm"], max_seqs, max_tokens, device, eps) for w in blocks]

    def close(self):
        self.closed = True
        self.first.close()
        for b in self.blocks:
            b.close()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def new_state(self, seqs=1):
        return SequenceState(self, seqs)

    def _forward(self, x, state, scan):
        import torch
        u, _ = self.first.run(x)
        h = x.to(torch.float32, copy=True)  # updated below: never the caller's x
        for b, window, s in zip(self.blocks, state.windows, state.states):
            p = b.in_proj.run(u)
            z, raw, dt = p[:, :b.inner], p[:, b.inner:b.inner + b.chans], p[:, b.inner + b.chans:]
            y = scan(b.scan, raw, dt, window, s)
            b.gate.run(y, gate=z, out=y)
            u, h = b.join.run(b.out_proj.run(y), residual=h, res_out=h)
        return u

    def run(self, x, state, offsets=None):
        """The normalised outputs [tokens, dim] of prompts in packed rows x
        (``offsets``: int32 device tensor of their first rows; none: of equal
        lengths), continuing from ``state``, which is brought up to date."""
        return self._forward(x, state, lambda op, raw, dt, w, s: op.run(
            raw, dt, w, s, window_out=w, state_out=s, seqs=state.seqs, offsets=offsets)[0])

    def step(self, x, state):
        """The same for one token per sequence, x [seqs, dim]."""
        return self._forward(x, state, lambda op, raw, dt, w, s: op.step(raw, dt, w, s, window_out=w, state_out=s)[0])

    def capture_step(self, state):
        """A captured HIP graph of ``step`` on ``state``: (x, y, replay), where x
        is filled with the tokens before each replay() and y holds their outputs
        after it.  ``state`` is as before the capture; its tensors are what every
        replay updates.  ``replay`` keeps the net and them alive, and refuses to
        run once the net is closed."""
        import torch
        with torch.cuda.device(self.device):
            x = torch.zeros(state.seqs, self.first.dim, dtype=self.first.torch_dtype, device=f"cuda:{self.device}")
            tensors = state.windows + state.states
            keep = [t.clone() for t in tensors]
            side = torch.cuda.Stream(self.device)
            side.wait_stream(torch.cuda.current_stream(self.device))
            with torch.cuda.stream(side):
                self.step(x, state)
            torch.cuda.current_stream(self.device).wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                y = self.step(x, state)
            for t, k in zip(tensors, keep):
                t.copy_(k)
        return x, y, _Replay(graph, self, tensors, (x, y))
