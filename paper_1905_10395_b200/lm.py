"""The operators of a language model's training step (include/lsgd.h), bound to torch tensors.

Each class takes the buffers that its operator works on once, checks them, and keeps the descriptor: a call afterwards is
one call of the C ABI, with no allocation and no synchronisation, so it can be captured in a CUDA graph.  The tensors must
outlive the object.  Work is enqueued on the stream given at construction (default: torch's current one at that time), not on
the one that is current at the call; a tensor last used on another stream has to be ordered with it by the caller.  An operator
that is to be captured is given the capture's stream: under a capture that its stream is not part of, a call is refused
(ERR_STATE).  The tensors' device has to be the current one at
every call (ERR_STATE otherwise).  There is no CPU path.  An operator has one scratch buffer: its calls, the replays of graphs that
captured it among them, run one after another (as they do on one stream); what is to run at once is given operators of its own.

Rows are [P, T, D] (worker, token, channel) with a channel stride of 1 and any row and worker stride; one worker's may be
given as [T, D].  Vectors are [P, D] or [D].  An input that is expanded over the workers (stride 0) is shared by them."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Union

import numpy as np
import torch

from . import api

_DTYPES = {torch.float32: api.F32, torch.bfloat16: api.BF16}
_current_device = torch._C._cuda_getDevice      # torch.cuda.current_device() without its check for initialisation: half the time
_current_stream = torch._C._cuda_getCurrentRawStream
_GATE_ACTS = {"identity": api.GATE_IDENTITY, "sigmoid": api.GATE_SIGMOID, "tanh": api.GATE_TANH}


def _fail(what: str) -> None:
    raise api.LsgdError(api.ERR_INVALID_ARG, what)


def _int32(name: str, v) -> int:
    """A size as a descriptor's 32-bit field holds it (ctypes would take a larger one modulo 2^32)."""
    v = int(v)
    if not -(1 << 31) <= v < 1 << 31:
        raise api.LsgdError(api.ERR_TOO_LARGE, f"{name}: {v}")
    return v


def _stream(stream, device: torch.device):
    """The stream that an operator keeps, for its calls and for the buffers that it allocates."""
    if stream is None:
        return torch.cuda.current_stream(device)
    if stream.device != device:
        _fail(f"a stream of {device}, got one of {stream.device}")
    return stream


def _not_left_out(stream, name: str) -> None:
    """Refuses a call under a capture that `stream` is not part of: the call would run at once and be missing from the graph."""
    if not torch.cuda.is_current_stream_capturing():
        return
    if stream.cuda_stream:                       # the default stream cannot be captured
        with torch.cuda.stream(stream):
            if torch.cuda.is_current_stream_capturing():
                return
    raise api.LsgdError(api.ERR_STATE, f"{name}: a capture is under way that the operator's stream is not part of")


def _dtype(name: str, *tensors) -> int:
    kinds = {t.dtype for t in tensors if t is not None}
    if len(kinds) > 1:
        _fail(f"{name}: one type is expected, got {sorted(map(str, kinds))}")
    for k in kinds:
        if k not in _DTYPES:
            raise api.LsgdError(api.ERR_UNSUPPORTED, f"{name}: {k}")
        return _DTYPES[k]
    return api.F32


def _same_device(*tensors) -> torch.device:
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1 or next(iter(devices)).type != "cuda":
        _fail(f"all tensors on one CUDA device, got {sorted(map(str, devices))}")
    return next(iter(devices))


def _rows(name: str, t: Optional[torch.Tensor], shape) -> api.Rows:
    """A [P, T, D] (or, for one worker, [T, D]) tensor as lsgd_rows."""
    if t is None:
        return api.Rows(None, 0, 0)
    if t.dim() == 2 and shape[0] == 1:
        t = t.unsqueeze(0)
    if tuple(t.shape) != tuple(shape):
        _fail(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.shape[2] > 1 and t.stride(2) != 1:
        _fail(f"{name}: the channels of a row have to be contiguous")
    return api.Rows(t.data_ptr() or None, t.stride(1), t.stride(0))


def _vector(name: str, t: Optional[torch.Tensor], P: int, D: int) -> api.Rows:
    """A [P, D] (or, for one worker, [D]) fp32 tensor as lsgd_rows of one row a worker."""
    if t is None:
        return api.Rows(None, 0, 0)
    if t.dim() == 1 and P == 1:
        t = t.unsqueeze(0)
    if tuple(t.shape) != (P, D):
        _fail(f"{name}: shape {tuple(t.shape)}, expected {(P, D)}")
    if t.dtype != torch.float32:
        raise api.LsgdError(api.ERR_UNSUPPORTED, f"{name}: {t.dtype}")
    if D > 1 and t.stride(1) != 1:
        _fail(f"{name}: the values of a vector have to be contiguous")
    return api.Rows(t.data_ptr() or None, 0, t.stride(0))


class _Bound:
    """A descriptor with its stream and what it points to."""

    def _bind(self, name, desc, device, stream, keep, scratch, *passes):
        """scratch: whether the operator needs any; passes: the directions whose sizes the library is asked for."""
        self.device, self._index, self._keep = device, device.index, [keep]
        self._stream, self._torch_stream = stream.cuda_stream, stream
        self._arg = stream.cuda_stream or None           # as the library gets it (None is passed on faster than 0)
        L = api.lib()
        self._forward, self._backward = getattr(L, f"lsgd_{name}_forward"), getattr(L, f"lsgd_{name}_backward")
        self._name, self.desc, self._ref = name, desc, C.byref(desc)
        if scratch:
            with torch.cuda.device(device):
                size = getattr(L, f"lsgd_{name}_scratch_bytes")
                n = max((int(size(self._ref, back)) for back in passes), default=0) if passes else int(size(self._ref))
            if n:
                with torch.cuda.stream(stream):      # the allocator's order of use is the operator's
                    buf = torch.empty(n, dtype=torch.uint8, device=device)
                desc.scratch, desc.scratch_bytes = buf.data_ptr(), n
                self._keep.append(buf)

    def _other_device(self) -> None:
        raise api.LsgdError(api.ERR_STATE, f"lsgd_{self._name}: device {_current_device()} is current, the tensors are on {self.device}")

    def forward(self) -> None:
        if _current_device() != self._index:     # the default stream would be the other device's, and so would the plan
            self._other_device()
        if _current_stream(self._index) != self._stream:
            _not_left_out(self._torch_stream, f"lsgd_{self._name}")
        s = self._forward(self._ref, self._arg)
        if s:
            raise api.LsgdError(s, f"lsgd_{self._name}_forward")

    def backward(self) -> None:
        if _current_device() != self._index:
            self._other_device()
        if _current_stream(self._index) != self._stream:
            _not_left_out(self._torch_stream, f"lsgd_{self._name}")
        s = self._backward(self._ref, self._arg)
        if s:
            raise api.LsgdError(s, f"lsgd_{self._name}_backward")


class Embedding(_Bound):
    """out[p, t] = scale * table[p, tokens[p, t]] (forward), and d_table from d_out (backward).

    tokens [P, T] int32 or int64; table, d_table [P, V, D]; out, d_out [P, T, D]; give the pair of each direction that is
    used.  d_table expanded over the workers sums over them.  accumulate: the gradient is added to d_table instead of
    replacing it.  padding: a token whose row gets no gradient (-1: none)."""

    def __init__(self, tokens: torch.Tensor, *, table: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 d_out: Optional[torch.Tensor] = None, d_table: Optional[torch.Tensor] = None, scale: float = 1.0,
                 padding: int = -1, accumulate: bool = False, stream=None):
        if tokens.dtype not in (torch.int32, torch.int64):
            raise api.LsgdError(api.ERR_UNSUPPORTED, f"tokens: {tokens.dtype}")
        tok = tokens.unsqueeze(0) if tokens.dim() == 1 else tokens
        if tok.dim() != 2 or (tok.shape[1] > 1 and tok.stride(1) != 1):
            _fail("tokens: [P, T] with the tokens of a worker contiguous")
        tables, acts = [t for t in (table, d_table) if t is not None], [t for t in (out, d_out) if t is not None]
        if not tables or (table is None) != (out is None) or (d_table is None) != (d_out is None):
            _fail("Embedding: table and out, or d_out and d_table, or all four")
        if any(t.dim() not in (2, 3) for t in tables):
            _fail("Embedding: tables of [P, V, D] or [V, D]")
        device = _same_device(tokens, *tables, *acts)
        stream = _stream(stream, device)
        P, T = tok.shape
        V, D = tables[0].shape[-2:]
        e = api.EmbedDesc()
        e.struct_size = C.sizeof(api.EmbedDesc)
        e.P, e.T, e.V, e.D = P, T, V, D
        e.token_bytes = tok.element_size()
        e.table_dtype, e.act_dtype = _dtype("table", *tables), _dtype("out", *acts)
        e.scale, e.padding, e.accumulate = float(scale), int(padding), int(accumulate)
        e.tokens, e.token_stride = tok.data_ptr() or None, tok.stride(0)
        e.table, e.out = _rows("table", table, (P, V, D)), _rows("out", out, (P, T, D))
        e.d_out, e.d_table = _rows("d_out", d_out, (P, T, D)), _rows("d_table", d_table, (P, V, D))
        self._bind("embed", e, device, stream, (tokens, table, out, d_out, d_table), d_table is not None)


class BlockNorm(_Bound):
    """The boundary between two blocks, x' = alpha x + beta a(gate) norm(y) w_post and h = norm(x') w_pre, and its gradient.

    x, out, d_out, dx [P, T, D] of the residual's type; y, h, d_h, dy of the activations'; gate, d_gate [P, D] fp32 (one
    value per channel) or [P, T, D] of the activations' type; w_post, w_pre, dw_post, dw_pre [P, D] fp32;
    rstd_post, rstd_pre [P, T] fp32, contiguous, written by forward and read by backward (allocated when not given).
    Without y only h is computed, and `out` of the backward pass is x.  Without w_pre there is no h."""

    def __init__(self, *, x: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                 w_pre: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None,
                 rstd_post: Optional[torch.Tensor] = None, rstd_pre: Optional[torch.Tensor] = None,
                 d_out: Optional[torch.Tensor] = None, d_h: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                 dy: Optional[torch.Tensor] = None, d_gate: Optional[torch.Tensor] = None,
                 dw_post: Optional[torch.Tensor] = None, dw_pre: Optional[torch.Tensor] = None, post_norm: bool = True,
                 gate_act: str = "identity", alpha: float = 1.0, beta: float = 1.0, eps: float = 1e-6,
                 accumulate: bool = False, stream=None):
        like = x if x is not None else out
        if like is None or like.dim() not in (2, 3):
            _fail("BlockNorm: x (or, for the backward pass alone, out) of [P, T, D] or [T, D]")
        P, T, D = like.shape if like.dim() == 3 else (1, *like.shape)
        if gate_act not in _GATE_ACTS:
            _fail(f"gate_act: one of {sorted(_GATE_ACTS)}")
        post_norm = bool(post_norm) and y is not None
        for given, of, names in (((h, d_h, dw_pre), w_pre, "h, d_h and dw_pre need w_pre"), ((d_gate,), gate, "d_gate needs a gate"),
                                 ((dy,), y, "dy needs y"), ((dw_post,), y if post_norm else None, "dw_post needs a norm of y")):
            if of is None and any(t is not None for t in given):
                _fail(f"BlockNorm: {names}")
        channel = gate is not None and gate.dim() == (2 if like.dim() == 3 else 1)
        token_gate = None if channel else gate
        keep = [x, y, gate, w_post, w_pre, out, h, rstd_post, rstd_pre, d_out, d_h, dx, dy, d_gate, dw_post, dw_pre]
        device = _same_device(*keep)
        stream = _stream(stream, device)
        d = api.BlocknormDesc()
        d.struct_size = C.sizeof(api.BlocknormDesc)
        d.P, d.T, d.D = P, T, D
        d.resid_dtype = _dtype("x", x, out, d_out, dx)
        acts = [t for t in (y, h, d_h, dy, token_gate, None if channel else d_gate) if t is not None]
        d.act_dtype = _dtype("y", *acts) if acts else d.resid_dtype
        d.post_norm, d.gate_act = int(post_norm), _GATE_ACTS[gate_act]
        d.gate_kind = api.GATE_NONE if gate is None else api.GATE_CHANNEL if channel else api.GATE_TOKEN
        d.alpha, d.beta, d.eps, d.accumulate = float(alpha), float(beta), float(eps), int(accumulate)
        full = (P, T, D)
        for name, t in (("x", x), ("y", y), ("out", out), ("h", h), ("d_out", d_out), ("d_h", d_h), ("dx", dx), ("dy", dy)):
            setattr(d, name, _rows(name, t, full))
        for name, t in (("gate", gate), ("d_gate", d_gate)):
            setattr(d, name, _vector(name, t, P, D) if channel else _rows(name, t, full))
        d.w_post, d.w_pre = _vector("w_post", w_post if post_norm else None, P, D), _vector("w_pre", w_pre, P, D)
        d.d_w_post, d.d_w_pre = _vector("dw_post", dw_post, P, D), _vector("dw_pre", dw_pre, P, D)
        stats = {}
        for name, t, used in (("rstd_post", rstd_post, post_norm), ("rstd_pre", rstd_pre, w_pre is not None)):
            if t is None and used:
                with torch.cuda.stream(stream):
                    t = torch.empty((P, T), dtype=torch.float32, device=device)
            if t is not None and (t.dtype != torch.float32 or t.numel() != P * T or not t.is_contiguous()):
                _fail(f"{name}: fp32 [P, T], contiguous")
            stats[name] = t
            setattr(d, name, (t.data_ptr() or None) if t is not None else None)
        self.rstd_post, self.rstd_pre = stats["rstd_post"], stats["rstd_pre"]
        keep += list(stats.values())
        self._bind("blocknorm", d, device, stream, keep, dx is not None)


def _given_rows(name: str, t: torch.Tensor):
    """[P, T, D] from a tensor of [P, T, D] or, for one worker, [T, D]."""
    if t.dim() not in (2, 3):
        _fail(f"{name}: [P, T, D] or [T, D]")
    return t if t.dim() == 3 else t.unsqueeze(0)


def _sequences(sequences: Optional[int], starts: Optional[torch.Tensor], P: int, T: int, device: torch.device) -> api.Sequences:
    if starts is None:
        S = 1 if sequences is None else _int32("sequences", sequences)
        if S < 1 or T % S:
            _fail(f"sequences: {S} equal parts of {T} rows")
        return api.Sequences(None, 0, S)
    if sequences is not None:
        _fail("sequences or starts, not both")
    if starts.dtype != torch.int32:
        raise api.LsgdError(api.ERR_UNSUPPORTED, f"starts: {starts.dtype}")
    if starts.device != device:
        _fail(f"starts: a tensor of {device}, got one of {starts.device}")
    if starts.dim() not in (1, 2) or starts.shape[-1] < 2 or (starts.dim() == 2 and starts.shape[0] != P) or starts.stride(-1) != 1:
        _fail("starts: [S + 1] or [P, S + 1], a worker's contiguous")
    S = _int32("starts", starts.shape[-1] - 1)
    return api.Sequences(starts.data_ptr(), starts.stride(0) if starts.dim() == 2 and P > 1 else 0, S)


def _table(name: str, t: Optional[torch.Tensor], P: int, rows: int, cols: int) -> api.Rows:
    """A [P, rows, cols] (or, for one worker, [rows, cols]) fp32 tensor as lsgd_rows."""
    if t is not None and t.dtype != torch.float32:
        raise api.LsgdError(api.ERR_UNSUPPORTED, f"{name}: {t.dtype}")
    return _rows(name, t, (P, rows, cols))


def _state(name: str, t: Optional[torch.Tensor], shape, dtype) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != dtype:
        raise api.LsgdError(api.ERR_UNSUPPORTED, f"{name}: {t.dtype}, expected {dtype}")
    if t.dim() == len(shape) - 1 and shape[0] == 1:
        t = t.unsqueeze(0)
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        _fail(f"{name}: contiguous {tuple(shape)}")
    return t.data_ptr() or None


class CausalConv(_Bound):
    """out[t] = act(bias + sum_j w[:, j] x[t - W + 1 + j]) along the sequences of every worker's rows, and its gradient.

    x, out, d_out, dx [P, T, D]; w, dw [P, D, W] and bias, d_bias [P, D], fp32 (gradients expanded over the workers are summed
    over them).  The T rows hold `sequences` sequences of equal length (default 1), or those whose first rows `starts` gives:
    int32 [S + 1] or [P, S + 1] on the device, ascending, the last entry the end of all; rows outside them are not touched.
    state [P, S, W - 1, D] of x's type: the inputs in front of every sequence, replaced by its last ones (forward only).
    act "silu" or "identity".  accumulate: dw and d_bias are added to."""

    def __init__(self, x: torch.Tensor, w: torch.Tensor, *, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 state: Optional[torch.Tensor] = None, d_out: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                 dw: Optional[torch.Tensor] = None, d_bias: Optional[torch.Tensor] = None, sequences: Optional[int] = None,
                 starts: Optional[torch.Tensor] = None, act: str = "silu", accumulate: bool = False, stream=None):
        if act not in ("silu", "identity"):
            _fail("act: silu or identity")
        device = _same_device(x, w, bias, out, state, d_out, dx, dw, d_bias)
        stream = _stream(stream, device)
        P, T, D = _given_rows("x", x).shape
        grads = any(t is not None for t in (d_out, dx, dw, d_bias))
        if grads and (d_out is None or dx is None or dw is None or (bias is None) != (d_bias is None)):
            _fail("CausalConv: the backward pass needs d_out, dx, dw and, with a bias, d_bias")
        if grads and state is not None:
            _fail("CausalConv: no gradient through a state")
        if out is None and not grads:
            _fail("CausalConv: out, or the tensors of the backward pass, or both")
        d = api.ConvDesc()
        d.struct_size = C.sizeof(api.ConvDesc)
        d.P, d.T, d.D, d.W = _int32("x", P), T, _int32("x", D), _int32("w", w.shape[-1])
        d.act_dtype = _dtype("x", x, out, d_out, dx)
        d.act, d.accumulate = (api.CONV_SILU if act == "silu" else api.CONV_IDENTITY), int(accumulate)
        d.seq = _sequences(sequences, starts, P, T, device)
        for name, t in (("x", x), ("out", out), ("d_out", d_out), ("dx", dx)):
            setattr(d, name, _rows(name, t, (P, T, D)))
        d.w, d.dw = _table("w", w, P, D, d.W), _table("dw", dw, P, D, d.W)
        d.bias, d.d_bias = _vector("bias", bias, P, D), _vector("d_bias", d_bias, P, D)
        d.state = _state("state", state, (P, d.seq.S, d.W - 1, D), x.dtype)
        passes = ([0] if out is not None else []) + ([1] if grads else [])
        self._bind("conv", d, device, stream, (x, w, bias, out, state, d_out, dx, dw, d_bias, starts), True, *passes)


class SelectiveScan(_Bound):
    """h[t] = exp(delta A) h[t - 1] + delta x[t] b[t],  y[t] = c[t] . h[t] + skip x[t],  out = y silu(z), with N states a channel,
    delta = softplus(dt + dt_bias) and A = -exp(a_log), along the sequences of every worker's rows; and its gradient.

    x, dt, z, out and their gradients [P, T, D]; b, c, d_b, d_c [P, T, N], all of one type; a_log, d_a_log [P, D, N] and skip,
    dt_bias and theirs [P, D], fp32 (gradients expanded over the workers are summed over them).  z, skip and dt_bias may be
    absent.  sequences / starts as for CausalConv.  state [P, S, D, N] fp32: what every sequence starts from, replaced by what it
    ends with (forward only; zeros without it).  saved [P, ceil(T / 8), D, N] fp32, written by forward and read by backward
    (allocated when not given; without `out`, which leaves the forward pass to another operator, that one's are given).  accumulate:
    d_a_log, d_skip and d_dt_bias are added to."""

    def __init__(self, x: torch.Tensor, dt: torch.Tensor, a_log: torch.Tensor, b: torch.Tensor, c: torch.Tensor, *,
                 z: Optional[torch.Tensor] = None, skip: Optional[torch.Tensor] = None, dt_bias: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, state: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                 d_out: Optional[torch.Tensor] = None, d_x: Optional[torch.Tensor] = None, d_dt: Optional[torch.Tensor] = None,
                 d_a_log: Optional[torch.Tensor] = None, d_b: Optional[torch.Tensor] = None, d_c: Optional[torch.Tensor] = None,
                 d_z: Optional[torch.Tensor] = None, d_skip: Optional[torch.Tensor] = None,
                 d_dt_bias: Optional[torch.Tensor] = None, sequences: Optional[int] = None, starts: Optional[torch.Tensor] = None,
                 accumulate: bool = False, stream=None):
        keep = [x, dt, a_log, b, c, z, skip, dt_bias, out, state, saved, d_out, d_x, d_dt, d_a_log, d_b, d_c, d_z, d_skip, d_dt_bias]
        device = _same_device(*keep)
        stream = _stream(stream, device)
        P, T, D = _given_rows("x", x).shape
        N = a_log.shape[-1]
        grads = any(t is not None for t in (d_out, d_x, d_dt, d_a_log, d_b, d_c, d_z, d_skip, d_dt_bias))
        if grads:
            if any(t is None for t in (d_out, d_x, d_dt, d_a_log, d_b, d_c)):
                _fail("SelectiveScan: the backward pass needs d_out, d_x, d_dt, d_a_log, d_b and d_c")
            for name, t, g in (("z", z, d_z), ("skip", skip, d_skip), ("dt_bias", dt_bias, d_dt_bias)):
                if (t is None) != (g is None):
                    _fail(f"SelectiveScan: {name} and its gradient are given together")
            if state is not None:
                _fail("SelectiveScan: no gradient through a state")
        if out is None and not grads:
            _fail("SelectiveScan: out, or the tensors of the backward pass, or both")
        d = api.ScanDesc()
        d.struct_size = C.sizeof(api.ScanDesc)
        d.P, d.T, d.D, d.N = _int32("x", P), T, _int32("x", D), _int32("a_log", N)
        d.act_dtype = _dtype("x", x, dt, b, c, z, out, d_out, d_x, d_dt, d_b, d_c, d_z)
        d.accumulate = int(accumulate)
        d.seq = _sequences(sequences, starts, P, T, device)
        for name, field, t in (("x", "x", x), ("dt", "dt", dt), ("z", "z", z), ("out", "out", out), ("d_out", "d_out", d_out),
                               ("d_x", "dx", d_x), ("d_dt", "d_dt", d_dt), ("d_z", "dz", d_z)):
            setattr(d, field, _rows(name, t, (P, T, D)))
        for name, field, t in (("b", "b", b), ("c", "c", c), ("d_b", "db", d_b), ("d_c", "dc", d_c)):
            setattr(d, field, _rows(name, t, (P, T, N)))
        d.a_log, d.d_a_log = _table("a_log", a_log, P, D, N), _table("d_a_log", d_a_log, P, D, N)
        for name, t in (("skip", skip), ("dt_bias", dt_bias), ("d_skip", d_skip), ("d_dt_bias", d_dt_bias)):
            setattr(d, name, _vector(name, t, P, D))
        d.state = _state("state", state, (P, d.seq.S, D, N), torch.float32)
        shape = (P, (T + api.SAVED_EVERY - 1) // api.SAVED_EVERY, D, N)
        if saved is None and grads:
            if out is None and T:
                _fail("SelectiveScan: a backward pass without a forward one (out) needs the saved states of that pass")
            with torch.cuda.stream(stream):
                saved = torch.empty(shape, dtype=torch.float32, device=device)
        d.saved = _state("saved", saved, shape, torch.float32)
        self.saved = saved
        passes = ([0] if out is not None else []) + ([1] if grads else [])
        self._bind("scan", d, device, stream, (*keep, saved, starts), True, *passes)


class Orthogonalize:
    """out = scale X, X the update of every worker's m x n matrix brought near an orthogonal one by Newton-Schulz products:
    X = U / (|U| + eps), then `steps` times X <- a X + (b G + c G G) X with G = X X^T.

    grad [P, m, n] (or [m, n]) fp32 or bf16; out the same in bf16.  momentum, fp32: M <- mu M + grad, in place, and U = M, or
    grad + mu M with nesterov; without it U = grad.  The products run on fp16 operands with a power-of-two scale, and carry what X is
    rounded by from step to step: with these coefficients and steps a result is within 0.4 % of its matrix's norm of the exact one,
    whatever its rank (0.2 % of full rank; 0.17 % is the rounding to bf16; of a few values up to 1 %, for their roundings do not
    average out)."""

    def __init__(self, grad: torch.Tensor, out: torch.Tensor, *, momentum: Optional[torch.Tensor] = None, mu: float = 0.95,
                 nesterov: bool = True, steps: int = 5, coefficients: Sequence[float] = (3.4445, -4.7750, 2.0315),
                 scale: float = 1.0, eps: float = 1e-7, stream=None):
        device = _same_device(grad, out, momentum)
        stream = _stream(stream, device)
        P, m, n = _given_rows("grad", grad).shape
        if out.dtype != torch.bfloat16:
            raise api.LsgdError(api.ERR_UNSUPPORTED, f"out: {out.dtype}")
        if len(coefficients) != 3:
            _fail("coefficients: a, b, c")
        d = api.OrthoDesc()
        d.struct_size = C.sizeof(api.OrthoDesc)
        d.P, d.m, d.n, d.steps, d.nesterov = _int32("grad", P), _int32("grad", m), _int32("grad", n), _int32("steps", steps), int(bool(nesterov))
        d.grad_dtype = _dtype("grad", grad)
        d.a, d.b, d.c = (float(v) for v in coefficients)
        d.mu, d.eps, d.scale = float(mu), float(eps), float(scale)
        d.grad, d.out = _rows("grad", grad, (P, m, n)), _rows("out", out, (P, m, n))
        d.momentum = _table("momentum", momentum, P, m, n)
        L = api.lib()
        self.device, self._index, self._keep = device, device.index, [grad, out, momentum]
        self._stream, self._torch_stream = stream.cuda_stream, stream
        self._arg = stream.cuda_stream or None
        self.desc, self._ref, self._call = d, C.byref(d), L.lsgd_ortho
        with torch.cuda.device(device):
            size = int(L.lsgd_ortho_scratch_bytes(self._ref))
        if size:
            with torch.cuda.stream(stream):          # the allocator's order of use is the operator's
                buf = torch.empty(size, dtype=torch.uint8, device=device)
            d.scratch, d.scratch_bytes = buf.data_ptr(), size
            self._keep.append(buf)

    def forward(self) -> None:
        if _current_device() != self._index:
            raise api.LsgdError(api.ERR_STATE, f"lsgd_ortho: device {_current_device()} is current, the tensors are on {self.device}")
        if _current_stream(self._index) != self._stream:
            _not_left_out(self._torch_stream, "lsgd_ortho")
        s = self._call(self._ref, self._arg)
        if s:
            raise api.LsgdError(s, "lsgd_ortho")

    def check(self) -> None:
        """Waits for the device and raises (ERR_DEVICE_FLAG) if a wait of the products' kernels ran out since it was last asked, of any
        operator on this device: what such a call left in `out` is not its result."""
        with torch.cuda.device(self.device):
            flag = api.lsgd_ortho_check_device()
        if flag:
            raise api.LsgdError(api.ERR_DEVICE_FLAG, f"lsgd_ortho: status {flag:#x}")


class AdamW:
    """One AdamW step over many tensors, in one launch.  params fp32, grads fp32 or bf16 (all of one type), each of them
    contiguous; copies: bf16 copies of the parameters (entries may be None), rewritten by every step.

    state "f32" or "8bit".  The moments m, v (and, for 8 bits, their block scales) are zeros, or given all together: flat buffers in
    which every tensor begins at a multiple of 256 values (`api.adamw_state_values` is their length; m, v fp32 or uint8,
    m_scale, v_scale fp32 of a 256th of it).  weight_decay: one number, or one for each tensor.  seed: of the random rounding
    of the 8-bit moments, which need an eps of at least 2^-50.  step: steps already taken (a restored run)."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *, state: Optional[str] = None,
                 m: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None, m_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None, copies: Optional[Sequence[Optional[torch.Tensor]]] = None,
                 beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.0, seed: int = 0, step: int = 0, stream=None):
        self.h = None
        params, grads = list(params), list(grads)
        n = len(params)
        if n == 0 or len(grads) != n or (copies is not None and len(copies) != n):
            _fail("AdamW: one gradient (and copy) for each of one or more tensors")
        copies = list(copies) if copies is not None else None
        for i, (p, g) in enumerate(zip(params, grads)):
            c = copies[i] if copies is not None else None
            if p.dtype != torch.float32:
                raise api.LsgdError(api.ERR_UNSUPPORTED, f"params[{i}]: {p.dtype}")
            if c is not None and c.dtype != torch.bfloat16:
                raise api.LsgdError(api.ERR_UNSUPPORTED, f"copies[{i}]: {c.dtype}")
            if g.numel() != p.numel() or (c is not None and c.numel() != p.numel()):
                _fail(f"AdamW: tensor {i} and its gradient or copy differ in size")
            if not p.is_contiguous() or not g.is_contiguous() or (c is not None and not c.is_contiguous()):
                _fail(f"AdamW: tensor {i} is not contiguous")
        grad_dtype = _dtype("grads", *grads)
        self.device = device = _same_device(*params, *grads, *[c for c in copies or [] if c is not None], m, v, m_scale, v_scale)
        self._stream = stream = _stream(stream, device)
        if state is None:
            state = "8bit" if m is not None and m.dtype == torch.uint8 else "f32"
        if state not in ("f32", "8bit"):
            _fail("state: f32 or 8bit")
        sizes = np.array([p.numel() for p in params], dtype=np.int64)
        self.values = values = api.adamw_state_values(sizes)
        kind = torch.uint8 if state == "8bit" else torch.float32

        def buffer(name, t, count, dtype):
            if t is None:
                with torch.cuda.stream(stream):      # cleared before the first step, on its stream
                    return torch.zeros(count, dtype=dtype, device=device)
            if t.dtype != dtype or t.numel() != count or not t.is_contiguous():
                _fail(f"{name}: {count} contiguous values of {dtype}")
            return t

        parts = (m, v, m_scale, v_scale) if state == "8bit" else (m, v)
        if any(t is not None for t in parts) and any(t is None for t in parts):
            _fail("AdamW: a state is given whole (m, v and, for 8 bits, m_scale and v_scale) or not at all")
        if state == "f32" and (m_scale is not None or v_scale is not None):
            _fail("AdamW: scales belong to 8-bit moments")
        self.m, self.v = buffer("m", m, values, kind), buffer("v", v, values, kind)
        self.m_scale = self.v_scale = None
        if state == "8bit":
            self.m_scale = buffer("m_scale", m_scale, values // 256, torch.float32)
            self.v_scale = buffer("v_scale", v_scale, values // 256, torch.float32)
        wd = np.ascontiguousarray(np.broadcast_to(np.asarray(weight_decay, dtype=np.float32), (n,)))
        ptrs = lambda ts: np.array([t.data_ptr() if t is not None else 0 for t in ts], dtype=np.uint64)  # noqa: E731
        host = [sizes, ptrs(params), ptrs(grads), ptrs(copies) if copies is not None else None, wd]
        d = api.AdamwDesc()
        d.struct_size, d.n_tensors = C.sizeof(api.AdamwDesc), n
        d.sizes, d.params, d.grads, d.copies, d.weight_decay = (a.ctypes.data if a is not None else None for a in host)
        d.grad_dtype, d.state_dtype = grad_dtype, api.STATE_8BIT if state == "8bit" else api.STATE_F32
        d.m, d.v = self.m.data_ptr(), self.v.data_ptr()
        if state == "8bit":
            d.m_scale, d.v_scale = self.m_scale.data_ptr(), self.v_scale.data_ptr()
        d.beta1, d.beta2, d.eps, d.seed = float(beta1), float(beta2), float(eps), int(seed) & 0xFFFFFFFF
        d.stream = stream.cuda_stream or None
        self.state = state
        self._keep = (params, grads, copies)
        h = C.c_void_p()
        with torch.cuda.device(device):
            s = api.lib().lsgd_adamw_create(C.byref(d), C.byref(h))
        if s:
            raise api.LsgdError(s, "lsgd_adamw_create")
        self.h = h
        self._step = api.lib().lsgd_adamw_step
        self._read = None
        if step:
            with torch.cuda.device(device):
                self.set_step(step)

    def _ready(self, name: str) -> None:
        if _current_stream(self.device.index) != self._stream.cuda_stream:
            _not_left_out(self._stream, name)

    def step(self, lr: float, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One step.  grad_scale: a device fp32 scalar that the gradients are multiplied by first."""
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or grad_scale.device != self.device):
            _fail("grad_scale: one fp32 value on the tensors' device")
        self._ready("lsgd_adamw_step")
        s = self._step(self.h, lr, grad_scale.data_ptr() if grad_scale is not None else None)
        if s:
            raise api.LsgdError(s, "lsgd_adamw_step")

    def moments(self):
        """The moments as the fp32 values that they stand for, flat, in buffers that the next call overwrites."""
        self._ready("lsgd_adamw_moments")
        if self._read is None:
            with torch.cuda.stream(self._stream):
                self._read = [torch.empty(self.values, dtype=torch.float32, device=self.device) for _ in range(2)]
        m, v = self._read
        s = api.lib().lsgd_adamw_moments(self.h, m.data_ptr(), v.data_ptr())
        if s:
            raise api.LsgdError(s, "lsgd_adamw_moments")
        return m, v

    def t(self) -> int:
        n = C.c_int64()
        s = api.lib().lsgd_adamw_get_step(self.h, C.byref(n))
        if s:
            raise api.LsgdError(s, "lsgd_adamw_get_step")
        return n.value

    def set_step(self, n: int) -> None:
        self._ready("lsgd_adamw_set_step")
        s = api.lib().lsgd_adamw_set_step(self.h, int(n))
        if s:
            raise api.LsgdError(s, "lsgd_adamw_set_step")

    def destroy(self) -> None:
        if self.h is not None:
            h, self.h = self.h, None
            api.lib().lsgd_adamw_destroy(h)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
