"""Python face of the sequence operators (sn_op handles of the C ABI).

Each class makes a handle from host weights (numpy arrays) and runs it on
device tensors: rows are the first dimension, rows may be strided (a slice of
a wider projection), elements of a row are contiguous.  A run enqueues on the
current stream of the handle's device, or on ``stream`` (a torch stream or a
stream's pointer), and returns at once.

With another stream than the current one, the caller has that stream wait for
what makes the tensors that are passed in, as with any work given to a stream.
Outputs that a run makes itself are that stream's: their memory has no earlier
use that the stream does not know of, and is not used again before the work
on it, and on the stream that was current, is done.
"""

from __future__ import annotations

import ctypes
import operator

import numpy as np

from . import native as N


def _f32(v, shape, name):
    """A float32 host array of the given shape, or None."""
    if v is None:
        return None
    a = np.ascontiguousarray(v, dtype=np.float32)
    if a.shape != tuple(shape):
        raise ValueError(f"{name} has shape {a.shape}, not {tuple(shape)}")
    return a


def _int(v, name, least=-(1 << 31)):
    """A whole number that fits the C ABI's int32 (ctypes would cut it to 32 bits)."""
    v = operator.index(v)
    if not least <= v < 1 << 31:
        raise ValueError(f"{name} is out of range: {v}")
    return v


def _fp(a):
    return None if a is None else a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))


class _Op:
    """A handle's lifetime, and what every run does with its tensors."""

    def __init__(self, dtype, device):
        import torch
        self._op = None
        self.lib = N.lib()
        self._torch = torch
        self._types = {N.F32: torch.float32, N.F16: torch.float16, N.BF16: torch.bfloat16}
        self.dtype = N.DTYPE[dtype] if isinstance(dtype, str) else dtype
        if self.dtype not in self._types:
            raise ValueError(f"unknown dtype {dtype!r}")
        self.torch_dtype = self._types[self.dtype]
        self.device = device = _int(device, "device")
        self._dev = torch.device("cuda", device) if device >= 0 else None
        # the current stream's pointer, without making a Stream object of it (1 us)
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)

    def close(self):
        if getattr(self, "_op", None):
            self.lib.sn_op_destroy(self._op)
            self._op = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _rows(self, t, name, rows, cols, dtype):
        """The row stride of a device tensor [rows, cols] that a kernel may use
        as it is.  (A call of a small operator is a few microseconds: the one
        test that all sound tensors pass comes first.)"""
        if t.dtype is dtype and t.get_device() == self.device and t.shape == (rows, cols):
            s, e = t.stride()
            if e == 1 or cols <= 1 or not rows:
                return s if rows > 1 else cols
            raise ValueError(f"the elements of a row of {name} are not contiguous")
        if t.dtype is not dtype:
            raise TypeError(f"{name} is {t.dtype}, not {dtype}")
        if t.shape != (rows, cols):
            raise ValueError(f"{name} has shape {tuple(t.shape)}, not {(rows, cols)}")
        raise ValueError(f"{name} is on {t.device}, the handle on {self._dev}")

    def _side(self, stream):
        """The stream to run on if it is another one than the current, else None."""
        if isinstance(stream, int):
            if stream == self._current(self.device):
                return None
            return self._torch.cuda.ExternalStream(stream, device=self._dev)
        return None if stream.cuda_stream == self._current(self.device) else stream

    def _new(self, x, shape, dtype, side):
        """An output on another stream: from the pool of the stream that writes it (a
        block of the current stream's may still be in use by work queued there)."""
        with self._torch.cuda.stream(side):
            t = x.new_empty(shape, dtype=dtype)
        t.record_stream(self._torch.cuda.current_stream(self.device))
        return t

    def _stream(self, side, tensors):
        """The pointer of another stream than the current one; the tensors' memory
        is kept from reuse until its work is done."""
        for t in tensors:
            if t is not None:
                t.record_stream(side)
        return side.cuda_stream


def quantize4(w, group=128, zero=False):
    """4-bit codes of a weight matrix [rows, cols]: (q, scale, zero points) as
    ``Linear4`` takes them, each group of ``group`` columns rounded to the
    nearest of 16 steps: symmetric around code 8, or with ``zero`` from the
    group's least to its largest value."""
    w = np.asarray(w, np.float32)
    rows, cols = w.shape
    groups = -(-cols // group)
    g = np.zeros((rows, groups * group), np.float32)
    g[:, :cols] = w
    g = g.reshape(rows, groups, group)
    if zero:
        lo, hi = np.minimum(g.min(2), 0), np.maximum(g.max(2), 0)
        scale = ((hi - lo) / 15).astype(np.float16)
    else:
        scale = (np.abs(g).max(2) / 7.5).astype(np.float16)
    scale = np.maximum(scale, np.float16(6.2e-5))  # no group's scale below the normal numbers
    step = scale.astype(np.float32)
    z = np.clip(np.rint(-lo / step), 0, 15).astype(np.uint8) if zero else None
    code = np.clip(np.rint(g / step[..., None]) + (8 if z is None else z[..., None]), 0, 15)
    code = code.reshape(rows, -1)[:, :cols + cols % 2].astype(np.uint8)
    if code.shape[1] % 2:
        code = np.pad(code, ((0, 0), (0, 1)))
    return code[:, 0::2] | (code[:, 1::2] << 4), scale, z


class Linear4(_Op):
    """Product with 4-bit weights: y[m, k] = act(sum_c x[m, c] * scale[k, c // group]
    * (q[k, c] - zero[k, c // group]) + bias[k]).

    ``q``: uint8 [rows, ceil(cols / 2)], feature 2j in the low half of byte j;
    ``scale``: float16 [rows, ceil(cols / group)]; ``zero``: uint8 codes 0 .. 15
    of the same shape, or None for 8; ``bias``: float32 [rows] or None;
    ``group``: a multiple of 32."""

    def __init__(self, dtype, q, scale, zero=None, bias=None, cols=None, group=128, act="none", device=0):
        super().__init__(dtype, device)
        q = np.ascontiguousarray(q, dtype=np.uint8)
        group = _int(group, "group", 1)
        self.rows = q.shape[0]
        self.cols = 2 * q.shape[1] if cols is None else _int(cols, "cols")
        if q.shape[1] != (self.cols + 1) // 2:
            raise ValueError(f"{q.shape[1]} bytes of codes a row do not hold {self.cols} columns")
        scale = np.ascontiguousarray(scale, dtype=np.float16)
        shape = (self.rows, -(-self.cols // group))
        if scale.shape != shape:
            raise ValueError(f"scale has shape {scale.shape}, not {shape}")
        if zero is not None:
            zero = np.ascontiguousarray(zero, dtype=np.uint8)
            if zero.shape != shape:
                raise ValueError(f"zero has shape {zero.shape}, not {shape}")
        bias = _f32(bias, (self.rows,), "bias")
        d = N.Linear4Desc(self.dtype, self.rows, self.cols, group, N.ACT[act])
        p = ctypes.c_void_p()
        N.check(self.lib.sn_qlinear_create(ctypes.byref(d), q.ctypes.data, scale.ctypes.data,
                                           None if zero is None else zero.ctypes.data, _fp(bias), device,
                                           ctypes.byref(p)))
        self._op, self._run = p, self.lib.sn_qlinear_run

    def run(self, x, out=None, stream=None):
        """Enqueue on x [m, cols]; returns y [m, rows]."""
        m = x.shape[0]
        xs = self._rows(x, "x", m, self.cols, self.torch_dtype)
        side = None if stream is None else self._side(stream)
        if out is None:
            shape, ys = (m, self.rows), self.rows
            out = x.new_empty(shape) if side is None else self._new(x, shape, x.dtype, side)
        else:
            ys = self._rows(out, "out", m, self.rows, self.torch_dtype)
        st = self._current(self.device) if side is None else self._stream(side, (x, out))
        rc = self._run(self._op, m, x.data_ptr(), xs, out.data_ptr(), ys, st)
        if rc:
            N.check(rc)
        return out


class Scan(_Op):
    """Selective state space scan with its short causal convolution.

    A token's row of ``x`` holds ``chans`` = heads * head_dim + 2 * groups *
    state raw values, its row of ``dt`` one raw step size per head.  With
    u_t = silu(conv_b + sum_j conv_w[:, j] * raw_{t - conv + 1 + j}) = [X | B | C]
    and dt_t = log(1 + exp(dt_raw_t + dt_bias)), each head computes::

        h_t = exp(dt_t * a) * h_{t-1} + dt_t * X_t (outer) B_t
        y_t = h_t C_t + d * X_t

    ``window`` [seqs, conv - 1, chans] holds the raw values before the first
    token (oldest first), ``state`` [seqs, heads, head_dim, state] (float32)
    the h before it; None means zeros.  Both come back as they are after the
    last token, in ``window_out`` and ``state_out`` (which may be the inputs:
    updated in place).  The workspace holds calls of up to ``max_seqs``
    sequences and ``max_tokens`` rows in all; calls share it, so they must
    follow each other on one stream."""

    def __init__(self, dtype, heads, head_dim, groups, state, conv_w, conv_b=None, a=None, d=None, dt_bias=None,
                 max_seqs=1, max_tokens=1, device=0):
        super().__init__(dtype, device)
        heads, head_dim, groups, state, max_seqs = (
            _int(v, n) for v, n in ((heads, "heads"), (head_dim, "head_dim"), (groups, "groups"), (state, "state"),
                                    (max_seqs, "max_seqs")))
        self.heads, self.head_dim, self.groups, self.state = heads, head_dim, groups, state
        self.inner, self.chans = heads * head_dim, heads * head_dim + 2 * groups * state
        conv_w = np.ascontiguousarray(conv_w, dtype=np.float32)
        if conv_w.ndim != 2 or conv_w.shape[0] != self.chans:
            raise ValueError(f"conv_w has shape {conv_w.shape}, not ({self.chans}, taps)")
        self.conv = conv_w.shape[1]
        if a is None:
            raise ValueError("a is missing")
        arrays = [conv_w] + [_f32(v, (n,), s) for v, n, s in ((conv_b, self.chans, "conv_b"), (a, heads, "a"),
                                                             (d, heads, "d"), (dt_bias, heads, "dt_bias"))]
        desc = N.ScanDesc(self.dtype, heads, head_dim, groups, state, self.conv, max_seqs, max_tokens)
        p = ctypes.c_void_p()
        N.check(self.lib.sn_scan_create(ctypes.byref(desc), *[_fp(v) for v in arrays], device, ctypes.byref(p)))
        self._op = p
        self._io = N.ScanIO()  # one call's arguments: filled anew by every call
        self._io_ref = ctypes.byref(self._io)

    def _whole(self, t, name, shape, dtype):
        if t.dtype is dtype and t.shape == shape and t.get_device() == self.device and t.is_contiguous():
            return t.data_ptr()
        raise ValueError(f"{name} is not a contiguous {dtype} tensor {tuple(shape)} on {self._dev}")

    def _call(self, f, x, dt, window, state, window_out, state_out, seqs, offsets, out, stream):
        tokens, kind, f32 = x.shape[0], self.torch_dtype, self._torch.float32
        io = self._io
        io.seqs, io.tokens = seqs, tokens
        io.x_stride, io.x = self._rows(x, "x", tokens, self.chans, kind), x.data_ptr()
        io.dt_stride, io.dt = self._rows(dt, "dt", tokens, self.heads, kind), dt.data_ptr()
        wshape, sshape = (seqs, self.conv - 1, self.chans), (seqs, self.heads, self.head_dim, self.state)
        io.window = None if window is None else self._whole(window, "window", wshape, kind)
        io.state = None if state is None else self._whole(state, "state", sshape, f32)
        io.offsets = None if offsets is None else self._whole(offsets, "offsets", (seqs + 1,), self._torch.int32)
        side = None if stream is None else self._side(stream)
        if out is None:
            shape = (tokens, self.inner)
            out = x.new_empty(shape) if side is None else self._new(x, shape, kind, side)
            io.y_stride, io.y = self.inner, out.data_ptr()
        else:
            io.y_stride, io.y = self._rows(out, "out", tokens, self.inner, kind), out.data_ptr()
        if window_out is None:
            window_out = x.new_empty(wshape) if side is None else self._new(x, wshape, kind, side)
        if state_out is None:
            state_out = x.new_empty(sshape, dtype=f32) if side is None else self._new(x, sshape, f32, side)
        io.window_out = self._whole(window_out, "window_out", wshape, kind)
        io.state_out = self._whole(state_out, "state_out", sshape, f32)
        st = self._current(self.device) if side is None else self._stream(
            side, (x, dt, window, state, offsets, out, window_out, state_out))
        rc = f(self._op, self._io_ref, st)
        if rc:
            N.check(rc)
        return out, window_out, state_out

    def run(self, x, dt, window=None, state=None, window_out=None, state_out=None, seqs=None, offsets=None, out=None,
            stream=None):
        """Enqueue on the packed rows x [tokens, chans], dt [tokens, heads] of
        one or more sequences; returns (y [tokens, heads * head_dim], window,
        state).  ``offsets`` (int32 device tensor [seqs + 1]) gives their first
        rows; without it ``seqs`` (default: what window or state hold, else 1)
        sequences share the rows evenly."""
        if seqs is None:
            seqs = (offsets.shape[0] - 1 if offsets is not None else window.shape[0] if window is not None
                    else state.shape[0] if state is not None else 1)
        return self._call(self.lib.sn_scan_run, x, dt, window, state, window_out, state_out, seqs, offsets, out, stream)

    def step(self, x, dt, window=None, state=None, window_out=None, state_out=None, out=None, stream=None):
        """The same for one token of each of x.shape[0] sequences, in one kernel."""
        return self._call(self.lib.sn_scan_step, x, dt, window, state, window_out, state_out, x.shape[0], None, out,
                          stream)


class BlockNorm(_Op):
    """Norms before and after a block with its gate, scale and residual.

    ``run`` computes, in float32 and in one pass::

        t = x;  t *= silu(gate)                      # gate="before"
        t = norm(t) * post + post_bias               # in `groups` parts, if post is given
        t *= silu(gate)                              # gate="after"
        t *= scale                                   # number or vector
        res_out = residual + t                       # with a residual type
        y = norm(res_out or t) * pre + pre_bias      # if pre is given; else t without a residual

    ``kind`` is "rms" or "layer"; ``residual`` names the residual's element
    type (None: no residual)."""

    def __init__(self, dtype, dim, kind="rms", post=None, post_bias=None, pre=None, pre_bias=None, scale=None,
                 gate="none", groups=1, eps=1e-5, residual=None, device=0):
        super().__init__(dtype, device)
        rd = -1 if residual is None else N.DTYPE[residual] if isinstance(residual, str) else residual
        self.dim, self.gate = _int(dim, "dim"), gate
        self.res_dtype = None if rd < 0 else self._types[rd]
        self.has_y = pre is not None or rd < 0
        vector = scale is not None and np.ndim(scale) > 0
        arrays = [_f32(v, (dim,), n) for v, n in ((post, "post"), (post_bias, "post_bias"), (pre, "pre"),
                                                  (pre_bias, "pre_bias"), (scale if vector else None, "scale"))]
        d = N.NormDesc(self.dtype, rd, dim, _int(groups, "groups"), N.NORM[kind], N.GATE[gate], eps,
                       1.0 if scale is None or vector else float(scale))
        p = ctypes.c_void_p()
        N.check(self.lib.sn_norm_create(ctypes.byref(d), *[_fp(a) for a in arrays], device, ctypes.byref(p)))
        self._op, self._run = p, self.lib.sn_norm_run

    def run(self, x, gate=None, residual=None, out=None, res_out=None, stream=None):
        """Enqueue on x [rows, dim]; returns (y, res_out), None for the one that
        the handle does not have.  ``out`` may be x and ``res_out`` residual."""
        rows, dim, kind = x.shape[0], self.dim, self.torch_dtype
        xs = self._rows(x, "x", rows, dim, kind)
        gp = gs = rp = rs = op = os = yp = ys = 0
        side = None if stream is None else self._side(stream)
        if gate is not None:
            gp, gs = gate.data_ptr(), self._rows(gate, "gate", rows, dim, kind)
        if self.res_dtype is not None:
            if residual is not None:
                rp, rs = residual.data_ptr(), self._rows(residual, "residual", rows, dim, self.res_dtype)
            if res_out is None:
                shape, rkind, os = (rows, dim), self.res_dtype, dim
                res_out = x.new_empty(shape, dtype=rkind) if side is None else self._new(x, shape, rkind, side)
            else:
                os = self._rows(res_out, "res_out", rows, dim, self.res_dtype)
            op = res_out.data_ptr()
        elif residual is not None:
            raise ValueError("a residual given to a handle without one")
        if self.has_y:
            if out is None:
                shape, ys = (rows, dim), dim
                out = x.new_empty(shape) if side is None else self._new(x, shape, kind, side)
            else:
                ys = self._rows(out, "out", rows, dim, kind)
            yp = out.data_ptr()
        st = self._current(self.device) if side is None else self._stream(side, (x, gate, residual, out, res_out))
        rc = self._run(self._op, rows, x.data_ptr(), xs, gp, gs, rp, rs, op, os, yp, ys, st)
        if rc:
            N.check(rc)
        return out, res_out
