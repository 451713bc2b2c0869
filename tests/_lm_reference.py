"""Plain 64-bit restatements of the language-model operators (include/lsgd.h), on the CPU, and guarded device buffers."""
import torch

F64 = torch.float64


# ---- block-boundary norms
def gate_act(z, act):
    return {"identity": z, "sigmoid": torch.sigmoid(z), "tanh": torch.tanh(z)}[act]


def norm(z, eps):
    return z / torch.sqrt(z.square().mean(-1, keepdim=True) + eps)


def blocknorm_forward(x, y=None, gate=None, w_post=None, w_pre=None, act="identity", alpha=1.0, beta=1.0, eps=1e-6):
    """(x', h) from float64 [P, T, D]; gate [P, D] or [P, T, D]; w [P, D]."""
    wide = lambda v: v if v.dim() == 3 else v[:, None]  # noqa: E731
    out = x
    if y is not None:
        u = y if w_post is None else norm(y, eps) * wide(w_post)
        out = alpha * x + beta * (u if gate is None else gate_act(wide(gate), act) * u)
    return out, None if w_pre is None else norm(out, eps) * wide(w_pre)


def blocknorm_backward(d_out, d_h, out, y=None, gate=None, w_post=None, w_pre=None, act="identity", alpha=1.0, beta=1.0, eps=1e-6):
    """Gradients by the formulas of the header: a dict of dx, dy, d_gate, dw_post, dw_pre, and (for bounds) the sums of the
    magnitudes that each weight gradient adds up."""
    wide = lambda v: v if v.dim() == 3 else v[:, None]  # noqa: E731
    got, size = {}, {}
    g = torch.zeros_like(out) if d_out is None else d_out
    if w_pre is not None:
        r = 1 / torch.sqrt(out.square().mean(-1, keepdim=True) + eps)
        n, up = out * r, d_h * wide(w_pre)
        got["dw_pre"], size["dw_pre"] = (d_h * n).sum(1), (d_h * n).abs().sum(1)
        g = g + r * (up - n * (up * n).mean(-1, keepdim=True))
    if y is None:
        return {"dx": g, **got}, size
    got["dx"] = alpha * g
    dz = beta * g
    n, r = y, None
    if w_post is not None:
        r = 1 / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
        n = y * r
    u = n if w_post is None else n * wide(w_post)
    if gate is not None:
        z = wide(gate)
        a = gate_act(z, act)
        slope = {"identity": torch.ones_like(a), "sigmoid": a * (1 - a), "tanh": 1 - a * a}[act]
        dg = dz * u * slope
        got["d_gate"] = dg if gate.dim() == 3 else dg.sum(1)
        size["d_gate"] = dg.abs() if gate.dim() == 3 else dg.abs().sum(1)
        dz = dz * a
    if w_post is None:
        got["dy"] = dz
        return got, size
    got["dw_post"], size["dw_post"] = (dz * n).sum(1), (dz * n).abs().sum(1)
    s = dz * wide(w_post)
    got["dy"] = r * (s - n * (s * n).mean(-1, keepdim=True))
    return got, size


# ---- embedding
def embed_forward(tokens, table, scale):
    """tokens [P, T], table float64 [P, V, D]; a token out of range gives zeros."""
    P, T = tokens.shape
    V = table.shape[1]
    out = torch.zeros((P, T, table.shape[2]), dtype=F64)
    for p in range(P):
        ok = (tokens[p] >= 0) & (tokens[p] < V)
        out[p, ok] = table[p, tokens[p, ok].long()] * scale
    return out


def embed_backward(tokens, d_out, V, scale, padding=-1):
    """(gradient [P, V, D], sum of the magnitudes added)."""
    P, T = tokens.shape
    grad = torch.zeros((P, V, d_out.shape[2]), dtype=F64)
    size = torch.zeros_like(grad)
    for p in range(P):
        ok = (tokens[p] >= 0) & (tokens[p] < V) & (tokens[p] != padding)
        grad[p].index_add_(0, tokens[p, ok].long(), d_out[p, ok] * scale)
        size[p].index_add_(0, tokens[p, ok].long(), (d_out[p, ok] * scale).abs())
    return grad, size


# ---- guarded device buffers: a matrix with any strides inside a larger allocation whose other words must not change
SENTINEL = {4: 0x7FA5A5A5, 2: 0x7FA5}
_WORD = {4: torch.int32, 2: torch.int16}


class Guarded:
    """A strided view of a device buffer; every word of the buffer that the view does not cover holds a pattern."""

    def __init__(self, shape, strides, dtype, offset=0, fill=None, pad=256):
        size = torch.empty((), dtype=dtype).element_size()
        span = sum((n - 1) * s for n, s in zip(shape, strides)) + 1 if all(shape) else 0
        self.raw = torch.full((pad + offset + span + pad,), SENTINEL[size], dtype=_WORD[size], device="cuda")
        self.view = torch.as_strided(self.raw.view(dtype), shape, strides, pad + offset)
        mine = torch.zeros_like(self.raw, dtype=torch.bool)
        torch.as_strided(mine, shape, strides, pad + offset).fill_(True)
        self.foreign = ~mine
        self.pattern = SENTINEL[size]
        if fill is not None and all(shape):
            self.view.copy_(fill)

    def intact(self):
        return bool((self.raw[self.foreign] == self.pattern).all())
