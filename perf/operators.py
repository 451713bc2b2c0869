"""The training operators around a language model's matrix products, as they are measured.

Three operators, for a population of P workers whose parameters are rows of one matrix:

  embed   out[p, t] = scale * table[p, token[p, t]], and the table's gradient, summed in fp32 over equal tokens;
  norm    x' = alpha x + beta a(gate) * norm(y) w_post,  h = norm(x') w_pre,  norm(z) = z / sqrt(mean z^2 + eps):
          the boundary between two blocks (either norm, the gate or the block's output may be absent), and its gradient;
  adamw   the AdamW step over many tensors at once, moments in 32 bits or in 8 bits with one scale per 256 values.

`own = False` runs the plain form below, `own = True` the kernels of this repository."""
import math

import torch

own = False

EPS = 1e-6                  # of the norms
ADAM = {"beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "lr": 1e-3, "weight_decay": 0.1}
BLOCK = 256                 # values that share a scale in the 8-bit states
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
U32 = 0xFFFFFFFF


# ------------------------------------------------------------------------------------------------ cases
def _embed(name, direction, P, T, V, D, table="f32", act="bf16", index="i32", pad=0.0, accumulate=False):
    return {"name": name, "op": "embed", "dir": direction, "P": P, "T": T, "V": V, "D": D, "table": table, "act": act,
            "index": index, "pad": pad, "accumulate": accumulate}


def _norm(name, direction, P, T, D, resid="bf16", act="bf16", y=True, post=True, gate="none", gate_act="identity", pre=True):
    return {"name": name, "op": "norm", "dir": direction, "P": P, "T": T, "D": D, "resid": resid, "act": act, "y": y,
            "post": post, "gate": gate, "gate_act": gate_act, "pre": pre}


def _adamw(name, P, D, L, V, state, grad, copy):
    return {"name": name, "op": "adamw", "P": P, "D": D, "L": L, "V": V, "state": state, "grad": grad, "copy": copy}


def listed():
    return [
        # one token of one worker, as a sampling loop looks it up: latency only
        _embed("embed one token", "forward", 1, 1, 32768, 1024),
        # a training step's lookup for eight workers, each in its own table
        _embed("embed 8 workers", "forward", 8, 4096, 16384, 1024),
        # the gradient of a short micro-batch added to a tied table's, which the output layer has already written
        _embed("embed grad short", "gradient", 1, 96, 8192, 512, act="f32", accumulate=True),
        # odd everything: three workers, a prime vocabulary, rows that no wide load fits, a third of the tokens padding
        _embed("embed grad odd", "gradient", 3, 1021, 10007, 250, table="bf16", index="i64", pad=0.33),
        # the gradient of a long batch, most of a large table untouched and a few tokens in thousands of places
        _embed("embed grad long", "gradient", 1, 65536, 50000, 2048, index="i64", pad=0.1),
        # one row, as a sampling loop crosses a block boundary: residual add and the next block's norm
        _norm("norm one row", "forward", 1, 1, 4096, post=False),
        # a training batch through a block boundary with both norms and a gate of its own for each value
        _norm("norm 8 workers", "forward", 8, 2048, 2048, resid="f32", gate="token", gate_act="sigmoid"),
        # its gradient, with a learned gate for each channel and bf16 throughout
        _norm("norm grad wide", "gradient", 1, 16384, 4096, gate="channel"),
        # odd rows in fp32, a tanh gate and no norm in front of the next block
        _norm("norm grad odd", "gradient", 5, 333, 1001, resid="f32", act="f32", gate="channel", gate_act="tanh", pre=False),
        # one worker's three-layer classifier (784-1024-1024-10): six tensors, states in 32 bits
        _adamw("adamw classifier", 1, 0, 0, 0, "f32", "f32", False),
        # a population of 32 of them, 192 tensors, with bf16 copies of the weights for the products
        _adamw("adamw population", 32, 0, 0, 0, "8bit", "bf16", True),
        # the tensors of one language-model worker of 0.4 billion parameters, states in 8 bits
        _adamw("adamw language model", 1, 2048, 6, 50000, "8bit", "bf16", True),
    ]


def _size(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; half of them odd or otherwise ragged."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and n >= 64:
        n = (n + 32) // 64 * 64
    return min(max(n, lo), hi)


def draw(rng):
    c = _draw(rng)
    return {k: v - 1 if k in "TVD" and v in (768, 3072) else v for k, v in c.items() if k != "name"}


def _draw(rng):
    op = rng.choice(("embed", "norm", "adamw"))
    if op == "embed":
        direction = rng.choice(("forward", "gradient"))
        P, V, D = rng.choice((1, 1, 2, 3, 8)), _size(rng, 16, 50000), _size(rng, 32, 4096)
        D = min(D, max(32, 100_000_000 // (P * V)))
        T = min(_size(rng, 1, 65536), max(1, 134_000_000 // (P * D)))
        return _embed("", direction, P, T, V, D, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")),
                      rng.choice(("i32", "i64")), rng.choice((0.0, 0.0, 0.2, 0.9)), direction == "gradient" and rng.random() < 0.3)
    if op == "norm":
        direction = rng.choice(("forward", "gradient"))
        P, D = rng.choice((1, 1, 2, 5, 8)), _size(rng, 32, 8192)
        T = min(_size(rng, 1, 65536), max(1, 67_000_000 // (P * D)))
        resid, act = rng.choice((("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")))
        y = rng.random() < 0.85
        gate = rng.choice(("none", "channel", "token")) if y else "none"
        return _norm("", direction, P, T, D, resid, act, y, y and rng.random() < 0.6, gate,
                     rng.choice(("identity", "sigmoid", "tanh")) if gate != "none" else "identity", not y or rng.random() < 0.8)
    state, grad, copy = rng.choice(("f32", "8bit")), rng.choice(("f32", "bf16")), rng.random() < 0.5
    if rng.random() < 0.3:
        return _adamw("", _size(rng, 1, 64), 0, 0, 0, state, grad, copy)
    P, D, L = rng.choice((1, 1, 2)), _size(rng, 17, 2048), _size(rng, 1, 12)
    V = min(_size(rng, 16, 50000), 90_000_000 // (P * D))
    while L > 1 and P * L * 12 * D * D > 220_000_000:
        L -= 1
    return _adamw("", P, D, L, V, state, grad, copy)


def _tensors(c):
    """(elements, decayed) of every tensor of one step: matrices are decayed, gains and biases are not."""
    if c["D"] == 0:
        one = [(784 * 1024, True), (1024, False), (1024 * 1024, True), (1024, False), (1024 * 10, True), (10, False)]
    else:
        D = c["D"]
        layer = [(D, False)] + [(D * D, True)] * 4 + [(D, False)] + [(4 * D * D, True)] * 2
        one = [(c["V"] * D, True)] + layer * c["L"] + [(D, False)]
    return one * c["P"]


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, shift=0.0):
        out = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(shift, scale, generator=gen)
        return out.to(dtype)

    c = case
    s = {"case": dict(c)}
    if c["op"] == "embed":
        P, T, V, D = c["P"], c["T"], c["V"], c["D"]
        # token k with a probability of about 1 / (k + 1), as words have it; each row's end is padding (token 0)
        u = torch.rand((P, T), generator=gen, device="cuda", dtype=torch.float64)
        tok = (torch.exp(u * math.log(V + 1)) - 1).floor().clamp_(0, V - 1).long()
        tok[:, T - int(T * c["pad"]):] = 0
        s["tokens"] = tok if c["index"] == "i64" else tok.int()
        s["scale"] = math.sqrt(D)
        s["padding"] = 0 if c["pad"] else -1
        if c["dir"] == "forward":
            s["table"] = normal(P, V, D, dtype=TYPES[c["table"]], scale=0.02)
            s["out"] = torch.empty((P, T, D), dtype=TYPES[c["act"]], device="cuda")
        else:
            s["d_out"] = normal(P, T, D, dtype=TYPES[c["act"]], scale=1e-3)
            s["d_table"] = normal(P, V, D, dtype=TYPES[c["table"]], scale=1e-2)
        return s
    if c["op"] == "norm":
        P, T, D = c["P"], c["T"], c["D"]
        R, A = TYPES[c["resid"]], TYPES[c["act"]]
        s["alpha"], s["beta"] = 1.0, (0.5 if c["gate"] != "none" else 1.0)
        if c["post"]:
            s["w_post"] = normal(P, D, scale=0.1, shift=1.0)
        if c["pre"]:
            s["w_pre"] = normal(P, D, scale=0.1, shift=1.0)
        if c["y"]:
            s["y"] = normal(P, T, D, dtype=A, scale=0.7)
        if c["gate"] == "channel":
            s["gate"] = normal(P, D, scale=0.3, shift=0.5)
        elif c["gate"] == "token":
            s["gate"] = normal(P, T, D, dtype=A)
        if c["dir"] == "forward":
            s["x"] = normal(P, T, D, dtype=R, scale=2.0)
            if c["y"]:
                s["out"] = torch.empty_like(s["x"])
            if c["pre"]:
                s["h"] = torch.empty((P, T, D), dtype=A, device="cuda")
            s["rstd_post"], s["rstd_pre"] = (torch.empty((P, T), device="cuda") for _ in range(2))
        else:
            s["out"] = normal(P, T, D, dtype=R, scale=2.0)      # x' of the forward pass (x itself without a block output)
            s["d_out"] = normal(P, T, D, dtype=R, scale=1e-3)
            s["dx"] = torch.empty_like(s["out"])
            if c["pre"]:
                s["d_h"] = normal(P, T, D, dtype=A, scale=1e-3)
                s["rstd_pre"] = torch.rsqrt(s["out"].float().square().mean(-1) + EPS)
                s["dw_pre"] = torch.empty_like(s["w_pre"])
            if c["y"]:
                s["dy"] = torch.empty_like(s["y"])
            if c["post"]:
                s["rstd_post"] = torch.rsqrt(s["y"].float().square().mean(-1) + EPS)
                s["dw_post"] = torch.empty_like(s["w_post"])
            if c["gate"] != "none":
                s["d_gate"] = torch.empty_like(s["gate"])
        return s
    # adamw: the tensors are pieces of one buffer, each begun at a multiple of 256 values; between them it is zero
    sizes = _tensors(c)
    starts, n = [], 0
    for size, _ in sizes:
        starts.append(n)
        n += (size + BLOCK - 1) // BLOCK * BLOCK
    blocks = n // BLOCK
    keep = torch.zeros(n, dtype=torch.bool, device="cuda")
    decay = torch.zeros(blocks, device="cuda")
    for at, (size, decayed) in zip(starts, sizes):
        keep[at:at + size] = True
        decay[at // BLOCK:(at + size + BLOCK - 1) // BLOCK] = ADAM["weight_decay"] if decayed else 0.0
    s["decay"] = decay
    # a tensor's gradients differ in size from row to row by a few orders of magnitude
    spread = torch.exp(normal(blocks, 1, scale=1.5) - 7.0)
    zero = torch.zeros((), device="cuda")
    s["x"] = torch.where(keep, normal(n, scale=0.02), zero)
    s["g"] = torch.where(keep, (normal(blocks, BLOCK) * spread).reshape(-1), zero).to(TYPES[c["grad"]])
    m = torch.where(keep, (normal(blocks, BLOCK) * (0.3 * spread)).reshape(-1), zero)
    v = torch.where(keep, (normal(blocks, BLOCK).square_().add_(0.1) * spread.square()).reshape(-1), zero)
    if c["state"] == "f32":
        s["m"], s["v"] = m, v
    else:
        half = torch.full((blocks, BLOCK), 1 << 19, dtype=torch.int64, device="cuda")
        s["m"], s["m_scale"] = _encode(m.view(blocks, BLOCK), half, 112, True)
        s["v"], s["v_scale"] = _encode(v.view(blocks, BLOCK), half, 96, False)
    s["copy"] = s["x"].to(torch.bfloat16) if c["copy"] else None
    s["sizes"], s["starts"] = [a for a, _ in sizes], starts
    s["step"], s["seed"] = 100, seed & U32
    return s


# ------------------------------------------------------------------------------------------------ plain form
def _embed_plain(s):
    c = s["case"]
    P, T, V, D = c["P"], c["T"], c["V"], c["D"]
    row = s["tokens"].long() + V * torch.arange(P, device="cuda")[:, None]
    if c["dir"] == "forward":
        return {"out": (s["table"].reshape(P * V, D)[row].float() * s["scale"]).to(TYPES[c["act"]])}
    d = s["d_out"].float() * s["scale"]
    if s["padding"] >= 0:
        d = torch.where((s["tokens"] == s["padding"])[..., None], 0.0, d)
    grad = torch.zeros((P * V, D), device="cuda").index_add_(0, row.reshape(-1), d.reshape(P * T, D)).view(P, V, D)
    if c["accumulate"]:
        grad += s["d_table"]
        s["d_table"].copy_(grad)
        return {"d_table": s["d_table"]}
    return {"d_table": grad.to(TYPES[c["table"]])}


_ACT = {"identity": lambda z: z, "sigmoid": lambda z: 1 / (1 + torch.exp(-z)), "tanh": lambda z: 2 / (1 + torch.exp(-2 * z)) - 1}
_SLOPE = {"identity": lambda a: torch.ones_like(a), "sigmoid": lambda a: a * (1 - a), "tanh": lambda a: 1 - a * a}


def _gate(s):
    c = s["case"]
    if c["gate"] == "none":
        return None
    a = _ACT[c["gate_act"]](s["gate"].float())
    return a[:, None] if c["gate"] == "channel" else a


def _norm_forward_plain(s):
    c, got = s["case"], {}
    xo = s["x"].float()
    if c["y"]:
        z = s["y"].float()
        if c["post"]:
            got["rstd_post"] = torch.rsqrt(z.square().mean(-1) + EPS)
            z = z * got["rstd_post"][..., None] * s["w_post"][:, None]
        a = _gate(s)
        if a is not None:
            z = z * a
        xo = s["alpha"] * xo + s["beta"] * z
        got["out"] = xo.to(TYPES[c["resid"]])
    if c["pre"]:
        got["rstd_pre"] = torch.rsqrt(xo.square().mean(-1) + EPS)
        got["h"] = (xo * got["rstd_pre"][..., None] * s["w_pre"][:, None]).to(TYPES[c["act"]])
    return got


def _norm_gradient_plain(s):
    c, got = s["case"], {}
    R, A = TYPES[c["resid"]], TYPES[c["act"]]
    d = s["d_out"].float()
    if c["pre"]:
        r = s["rstd_pre"][..., None]
        n = s["out"].float() * r
        t = s["d_h"].float()
        got["dw_pre"] = (t * n).sum(1)
        t = t * s["w_pre"][:, None]
        d = d + r * (t - n * (t * n).mean(-1, keepdim=True))
    if not c["y"]:
        return {"dx": d.to(R), **got}
    got["dx"] = (s["alpha"] * d).to(R)
    dz = s["beta"] * d
    u = s["y"].float()
    if c["post"]:
        n = u * s["rstd_post"][..., None]
        u = n * s["w_post"][:, None]
    a = _gate(s)
    if a is not None:
        dg = dz * u * _SLOPE[c["gate_act"]](a)
        got["d_gate"] = dg.sum(1) if c["gate"] == "channel" else dg.to(A)
        dz = dz * a
    if c["post"]:
        got["dw_post"] = (dz * n).sum(1)
        t = dz * s["w_post"][:, None]
        dz = s["rstd_post"][..., None] * (t - n * (t * n).mean(-1, keepdim=True))
    got["dy"] = dz.to(A)
    return got


# An 8-bit value is a small float: `code << 20` are the bits of an fp32 number whose exponent field begins at 0, so that
# 2^112 (4 bits of exponent, with a sign) or 2^96 (5 bits, without) times it is between 0 and 1.875, and a block's largest
# value is 1.875 of its scale.  The 20 bits below a code are rounded at random.
def _decode(code, scale, shift, signed):
    c = code.to(torch.int32)
    mag = ((c & 127 if signed else c) << 20).view(torch.float32) * 2.0 ** shift * scale[:, None]
    return torch.where(c > 127, -mag, mag) if signed else mag


def _encode(z, low, shift, signed):
    a = z.abs()
    top = a.amax(1)
    scale = torch.where(top >= 2.0 ** -100, top * 0.53333336, 0.0)
    inv = torch.where(scale > 0, 1 / scale, 0.0)
    bits = (a * inv[:, None] * 2.0 ** -shift).view(torch.int32).long()
    code = ((bits + low) >> 20).clamp_(max=127 if signed else 255)
    if signed:
        code = code + 128 * (z < 0)
    else:
        code = torch.maximum(code, (bits > 0).long())       # a second moment that is not zero is not rounded to zero
    return code.to(torch.uint8).view(-1), scale


def _mix(h):
    h = (h * 0x9E3779B1) & U32
    h = h ^ (h >> 15)
    h = (h * 0x85EBCA77) & U32
    return h ^ (h >> 13)


def _adamw_plain(s):
    c = s["case"]
    s["step"] += 1
    t = s["step"]
    b1, b2, lr = ADAM["beta1"], ADAM["beta2"], ADAM["lr"]
    n = s["x"].numel()
    g = s["g"].float()
    if c["state"] == "f32":
        m, v = s["m"], s["v"]
    else:
        m, v = _decode(s["m"].view(-1, BLOCK), s["m_scale"], 112, True), _decode(s["v"].view(-1, BLOCK), s["v_scale"], 96, False)
        g = g.view(-1, BLOCK)
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * (1 - b2) * g
    denom = v.sqrt() / math.sqrt(1 - b2 ** t) + ADAM["eps"]
    x = s["x"].view(-1, BLOCK)
    x = x * (1 - lr * s["decay"][:, None]) - (lr / (1 - b1 ** t)) * (m / denom).view(-1, BLOCK)
    s["x"].copy_(x.view(-1))
    if c["copy"]:
        s["copy"].copy_(s["x"])
    if c["state"] == "f32":
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        h = _mix(torch.arange(n, device="cuda").view(-1, BLOCK) ^ _mix(_mix(s["seed"]) ^ (t & U32)))
        s["m"], s["m_scale"] = _encode(m, (h & 0xFFFF) << 4, 112, True)
        s["v"], s["v_scale"] = _encode(v, (h >> 16) << 4, 96, False)
        m, v = _decode(s["m"].view(-1, BLOCK), s["m_scale"], 112, True), _decode(s["v"].view(-1, BLOCK), s["v_scale"], 96, False)
    return {"x": s["x"], "m": m.view(-1), "v": v.view(-1), **({"copy": s["copy"]} if c["copy"] else {})}


# ------------------------------------------------------------------------------------------------ the repository's kernels
def _own_op(s):
    """The bound operator that a user's program keeps beside its buffers: made at the first pass."""
    from paper_1905_10395_b200 import lm
    c = s["case"]
    if c["op"] == "embed":
        kw = {k: s[k] for k in ("table", "out", "d_out", "d_table") if k in s}
        return lm.Embedding(s["tokens"], scale=s["scale"], padding=s["padding"], accumulate=c["accumulate"], **kw)
    if c["op"] == "norm":
        names = ("x", "y", "gate", "w_post", "w_pre", "out", "h", "rstd_post", "rstd_pre", "d_out", "d_h", "dx", "dy", "d_gate",
                 "dw_post", "dw_pre")
        kw = {k: s[k] for k in names if k in s}
        return lm.BlockNorm(alpha=s["alpha"], beta=s["beta"], eps=EPS, gate_act=c["gate_act"], post_norm=c["post"], **kw)
    pieces = lambda flat: [flat[a:a + n] for a, n in zip(s["starts"], s["sizes"])]  # noqa: E731
    decay = s["decay"].cpu().tolist()
    return lm.AdamW(pieces(s["x"]), pieces(s["g"]), m=s["m"], v=s["v"], m_scale=s.get("m_scale"), v_scale=s.get("v_scale"),
                    copies=pieces(s["copy"]) if c["copy"] else None, beta1=ADAM["beta1"], beta2=ADAM["beta2"], eps=ADAM["eps"],
                    weight_decay=[decay[a // BLOCK] for a in s["starts"]], seed=s["seed"], step=s["step"])


def _run_own(s):
    c = s["case"]
    if "op" not in s:
        s["op"] = _own_op(s)
    op = s["op"]
    if c["op"] == "embed":
        if c["dir"] == "forward":
            op.forward()
            return {"out": s["out"]}
        op.backward()
        return {"d_table": s["d_table"]}
    if c["op"] == "norm":
        names = ("dx", "dw_pre", "dw_post", "d_gate", "dy")
        if c["dir"] == "forward":
            op.forward()
            names = (("out",) if c["y"] else ()) + (("rstd_post",) if c["post"] else ()) + (("h", "rstd_pre") if c["pre"] else ())
        else:
            op.backward()
        return {k: s[k] for k in names if k in s}
    op.step(ADAM["lr"])
    m, v = (s["m"], s["v"]) if c["state"] == "f32" else op.moments()
    return {"x": s["x"], "m": m, "v": v, **({"copy": s["copy"]} if c["copy"] else {})}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "embed":
        return _embed_plain(state)
    if c["op"] == "norm":
        return _norm_forward_plain(state) if c["dir"] == "forward" else _norm_gradient_plain(state)
    return _adamw_plain(state)


# ------------------------------------------------------------------------------------------------ work
def _distinct(c):
    """Expected number of different tokens of one worker."""
    k = torch.arange(c["V"], dtype=torch.float64)
    p = torch.log((k + 2) / (k + 1)) / math.log(c["V"] + 1)
    return float((1 - (1 - p) ** (c["T"] - int(c["T"] * c["pad"]))).sum())


def work(case):
    c = case
    if c["op"] == "embed":
        P, n, D = c["P"], c["P"] * c["T"], c["D"]
        kept = n - P * int(c["T"] * c["pad"])
        tb, ab = BYTES[c["table"]], BYTES[c["act"]]
        index = n * BYTES[c["index"]]
        if c["dir"] == "forward":
            return {"bytes": index + P * _distinct(c) * D * tb + n * D * ab, "flops": n * D}
        rows = 2 * P * _distinct(c) if c["accumulate"] else P * c["V"]
        return {"bytes": index + kept * D * ab + rows * D * tb, "flops": 2 * kept * D}
    if c["op"] == "norm":
        P, n, D = c["P"], c["P"] * c["T"], c["D"]
        r, a = BYTES[c["resid"]], BYTES[c["act"]]
        token, channel = c["gate"] == "token", c["gate"] == "channel"
        vectors = P * D * 4 * (c["post"] + c["pre"] + channel)
        stats = n * 4 * (c["post"] + c["pre"])
        if c["dir"] == "forward":
            each = r + a * c["pre"] + (a + r) * c["y"] + a * token
            return {"bytes": n * D * each + vectors + stats, "flops": 10 * n * D}
        each = 2 * r + (a + r) * c["pre"] + 2 * a * c["y"] + 2 * a * token
        return {"bytes": n * D * each + 2 * vectors + stats, "flops": 25 * n * D}
    n = sum(size for size, _ in _tensors(c))
    each = 8 + BYTES[c["grad"]] + (2 if c["copy"] else 0)
    # 8-bit moments are also read out as the fp32 values that they stand for
    each += 16 if c["state"] == "f32" else 4 + 16 / BLOCK + 8
    return {"bytes": n * each, "flops": 15 * n}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f = lambda k: s[k].to(torch.float64)  # noqa: E731
    c = case
    if c["op"] == "embed":
        tok = s["tokens"].long()
        if c["dir"] == "forward":
            return {"out": torch.stack([f("table")[p].index_select(0, tok[p]) for p in range(c["P"])]) * s["scale"]}
        got = []
        for p in range(c["P"]):     # sorted by token, so that a token's gradient is the difference of two running sums' ends
            order = torch.argsort(tok[p], stable=True)
            live = order[tok[p][order] != s["padding"]]
            ids, counts = torch.unique_consecutive(tok[p][live], return_counts=True)
            grad = f("d_table")[p] if c["accumulate"] else torch.zeros((c["V"], c["D"]), dtype=torch.float64, device="cuda")
            if ids.numel():
                rows = s["d_out"][p].index_select(0, live).to(torch.float64)
                grad[ids] += s["scale"] * torch.segment_reduce(rows, "sum", lengths=counts)
            got.append(grad)
        return {"d_table": torch.stack(got)}
    if c["op"] == "norm":
        act = {"identity": lambda z: z, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[c["gate_act"]]
        shape = lambda z: z if z.dim() == 3 else z.unsqueeze(1)  # noqa: E731
        root = lambda z: 1 / torch.sqrt(z.pow(2).sum(-1, keepdim=True) / c["D"] + EPS)  # noqa: E731
        got = {}
        if c["dir"] == "forward":
            res = f("x")
            if c["y"]:
                b = f("y")
                if c["post"]:
                    got["rstd_post"] = root(b).squeeze(-1)
                    b = root(b) * b * shape(f("w_post"))
                if c["gate"] != "none":
                    b = act(shape(f("gate"))) * b
                res = s["alpha"] * res + s["beta"] * b
                got["out"] = res
            if c["pre"]:
                got["rstd_pre"] = root(res).squeeze(-1)
                got["h"] = root(res) * res * shape(f("w_pre"))
            return got
        # the gradient by the chain rule through h = r z w, with r the reciprocal root that the forward pass kept

        def through(z, r, up):
            r = r.unsqueeze(-1)
            return r * up - r.pow(3) / c["D"] * z * (up * z).sum(-1, keepdim=True)

        d = f("d_out")
        if c["pre"]:
            got["dw_pre"] = (f("d_h") * f("out") * f("rstd_pre").unsqueeze(-1)).sum(1)
            d = d + through(f("out"), f("rstd_pre"), f("d_h") * shape(f("w_pre")))
        if not c["y"]:
            return {"dx": d, **got}
        got["dx"] = s["alpha"] * d
        d = s["beta"] * d
        b = f("y")
        normed = b * f("rstd_post").unsqueeze(-1) if c["post"] else b
        gained = normed * shape(f("w_post")) if c["post"] else b
        if c["gate"] != "none":
            z = shape(f("gate"))
            slope = {"identity": torch.ones_like(z), "sigmoid": torch.sigmoid(z) * torch.sigmoid(-z), "tanh": torch.cosh(z).pow(-2)}[c["gate_act"]]
            dg = d * gained * slope
            got["d_gate"] = dg.sum(1) if c["gate"] == "channel" else dg
            d = d * act(z)
        if c["post"]:
            got["dw_post"] = (d * normed).sum(1)
            d = through(b, f("rstd_post"), d * shape(f("w_post")))
        got["dy"] = d
        return got
    # adamw: the definition, with the parameters' step in 64 bits.  The stored 8-bit moments are the rounding of a number
    # with 20 more bits than they keep by given random bits; they are rounded here from the moments in 64 bits.
    n = s["x"].numel()
    t = s["step"] + 1
    b1, b2 = ADAM["beta1"], ADAM["beta2"]
    if c["state"] == "f32":
        m, v = f("m"), f("v")
    else:
        def small(code, lead, bias):     # value of a code: subnormal below the first full exponent
            e, k = (code // 8).double(), (code % 8).double()
            return torch.where(e == 0, k / 8 * 2.0 ** (1 - bias), (1 + k / 8) * torch.exp2(e - bias)) * lead
        cm, cv = s["m"].long().view(-1, BLOCK), s["v"].long().view(-1, BLOCK)
        sign = 1.0 - 2.0 * (cm // 128).double()
        m = (small(cm % 128, sign, 15) * f("m_scale")[:, None]).view(-1)
        v = (small(cv, 1.0, 31) * f("v_scale")[:, None]).view(-1)
    g = f("g")
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    decay = f("decay").repeat_interleave(BLOCK)
    x = f("x")
    x = x - ADAM["lr"] * decay * x - ADAM["lr"] * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + ADAM["eps"])
    if c["state"] == "8bit":
        def mixed(h):
            h = h * 0x9E3779B1 % 2 ** 32
            h = h ^ h // 2 ** 15
            h = h * 0x85EBCA77 % 2 ** 32
            return h ^ h // 2 ** 13

        h = torch.arange(n, device="cuda") ^ mixed(mixed(s["seed"]) ^ t)
        h = torch.remainder(h * 0x9E3779B1, 2 ** 32)
        h = h ^ h // 2 ** 15
        lo = (h % 2 ** 16 * (0x85EBCA77 % 2 ** 32) + (h // 2 ** 16 * 0x85EBCA77 % 2 ** 16) * 2 ** 16) % 2 ** 32
        h = lo ^ lo // 2 ** 13
        for name in ("m", "v"):
            z, bias = (m, 15) if name == "m" else (v, 31)
            part = (h % 2 ** 16 if name == "m" else h // 2 ** 16).double() / 2 ** 16
            z = z.view(-1, BLOCK)
            scale = z.abs().amax(1, keepdim=True) / 1.875
            q = torch.where(scale > 0, z.abs() / scale, 0.0)
            e = torch.frexp(q)[1].clamp_(min=2 - bias) - 1              # of the value's binade, or of the first full one
            units = torch.ldexp(q, 3 - e)                                # in steps of a code there: 8 to 16, below 8 if subnormal
            low = torch.floor(units)
            up = low + (units - low + part.view(-1, BLOCK) >= 1)
            value = torch.ldexp(up, e - 3)
            if name == "v":
                value = torch.where((q > 0) & (value == 0), 2.0 ** (-2 - bias), value)
            value = value.clamp_(max=1.875) * torch.sign(z) * scale
            if name == "m":
                m = value.view(-1)
            else:
                v = value.view(-1)
    return {"x": x, "m": m, "v": v, **({"copy": x} if c["copy"] else {})}
