"""The operators of a language model's training step (include/lsgd.h), bound to torch tensors.

Each class takes the buffers that its operator works on once, checks them, and keeps the descriptor: a call afterwards is
one call of the C ABI, with no allocation and no synchronisation, so it can be captured in a CUDA graph.  The tensors must
outlive the object.  Work is enqueued on the stream given at construction (default: torch's current one at that time), not on
the one that is current at the call; a tensor last used on another stream has to be ordered with it by the caller.  An operator
that is to be captured is given the capture's stream: under a capture that its stream is not part of, a call is refused
(ERR_STATE).  The tensors' device has to be the current one at
every call (ERR_STATE otherwise).  There is no CPU path.

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

    def _bind(self, name, desc, device, stream, keep, scratch):
        self.device, self._index, self._keep = device, device.index, [keep]
        self._stream, self._torch_stream = stream.cuda_stream, stream
        self._arg = stream.cuda_stream or None           # as the library gets it (None is passed on faster than 0)
        L = api.lib()
        self._forward, self._backward = getattr(L, f"lsgd_{name}_forward"), getattr(L, f"lsgd_{name}_backward")
        self._name, self.desc, self._ref = name, desc, C.byref(desc)
        if scratch:
            with torch.cuda.device(device):
                n = int(getattr(L, f"lsgd_{name}_scratch_bytes")(self._ref))
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
