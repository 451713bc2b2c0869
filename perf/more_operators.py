"""A language model's recurrent mixer and its matrices' optimiser step, as they are measured.

Three operators, for a population of P workers whose sequences lie one behind another in rows [P, T, D] (worker, token, channel):

  conv    out_t = act(bias + sum_j w_j x_(t - W + 1 + j)): a short causal convolution of every channel, of a sequence's own
          tokens and, where a state is kept, of the W - 1 inputs before them; and its gradient;
  scan    h_t = exp(delta_t A) h_(t-1) + delta_t x_t B_t,  y_t = C_t . h_t + skip x_t,  out = y silu(z), with N states a
          channel, delta = softplus(dt + dt_bias) and A = -exp(a_log): a selective state space scan, and its gradient;
  ortho   X <- a X + (b G + c G G) X with G = X X^T, from X = U / |U|: the update U of a matrix (a gradient, or its momentum)
          brought near an orthogonal matrix by Newton-Schulz products.

Sequences are given by their starts (S + 1 of them a worker, the last one the end of all), or are S equal parts of the T tokens.
Rows in front of the first and behind the last sequence are not touched.  `own = False` runs the plain form below, `own = True` the
kernels of this repository."""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7     # of the products
MU = 0.95                                                 # of the momentum


# ------------------------------------------------------------------------------------------------ cases
def _conv(name, direction, P, T, S, D, W=4, act="bf16", silu=True, ragged=False, state=False):
    return {"name": name, "op": "conv", "dir": direction, "P": P, "T": T, "S": S, "D": D, "W": W, "act": act, "silu": silu,
            "ragged": ragged, "state": state}


def _scan(name, direction, P, T, S, D, N=16, act="bf16", gate=True, ragged=False, state=False):
    return {"name": name, "op": "scan", "dir": direction, "P": P, "T": T, "S": S, "D": D, "N": N, "act": act, "gate": gate,
            "ragged": ragged, "state": state}


def _ortho(name, P, m, n, grad="f32", momentum=True):
    return {"name": name, "op": "ortho", "P": P, "m": m, "n": n, "grad": grad, "momentum": momentum}


def listed():
    return [
        # the next token of one sequence: latency only
        _conv("conv one token", "forward", 1, 1, 1, 2048, state=True),
        # prompts of seven sequences of any length, packed, whose last inputs are kept for the tokens to come
        _conv("conv prompts", "forward", 1, 8191, 7, 4096, ragged=True, state=True),
        # a training step's convolution for eight workers, two sequences each: forward and gradient
        _conv("conv training", "training", 8, 2048, 2, 2048),
        # the next token of 64 sequences: the states are read and written
        _scan("scan 64 tokens", "forward", 1, 64, 64, 4096, state=True),
        # packed prompts, an odd number of channels, states kept for the tokens to come
        _scan("scan prompts", "forward", 1, 8191, 7, 1500, ragged=True, state=True),
        # a training step's scan for eight workers: forward and gradient
        _scan("scan training", "training", 8, 2048, 1, 2048),
        # one long sequence of a narrow model in fp32: the work has to be split over time
        _scan("scan training long", "training", 1, 32768, 1, 384, act="f32", gate=False),
        # odd everything: ragged sequences (some empty), channels that no wide load fits, 11 states
        _scan("scan training odd", "training", 3, 1021, 5, 250, N=11, act="f32", ragged=True),
        # eight small language models' first products (128 x 128): all steps of a matrix fit one SM
        _ortho("ortho small", 8, 128, 128),
        # the second matrix (1024 x 1024) of a population of 32 three-layer classifiers
        _ortho("ortho classifiers", 32, 1024, 1024),
        # three tall matrices of odd sizes
        _ortho("ortho odd", 3, 1001, 333, grad="bf16"),
        # one wide matrix of a larger model, from a bf16 gradient without momentum
        _ortho("ortho wide", 1, 2048, 8192, grad="bf16", momentum=False),
    ]


def _size(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; half of them odd or otherwise ragged."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and n >= 64:
        n = (n + 32) // 64 * 64
    return min(max(n, lo), hi)


def draw(rng):
    op = rng.choice(("conv", "scan", "scan", "ortho"))
    if op == "ortho":
        P, m, n = rng.choice((1, 1, 2, 3, 8, 32)), _size(rng, 16, 2048), _size(rng, 16, 8192)
        least = min(m, n)
        while P > 1 and P * least * least * (3 * max(m, n) + least) > 1.3e11:
            P -= 1
        c = _ortho("", P, m, n, rng.choice(("f32", "bf16")), rng.random() < 0.6)
        if rng.random() < 0.5:
            c["m"], c["n"] = n, m
        return {k: v for k, v in c.items() if k != "name"}
    direction = rng.choice(("forward", "training"))
    P, D, act = rng.choice((1, 1, 2, 3, 8)), _size(rng, 17, 4096), rng.choice(("bf16", "f32"))
    if op == "conv":
        T = min(_size(rng, 1, 32768), max(1, 33_000_000 // (P * D)))
    else:
        N = rng.choice((16, 16, 8, 32, 64, 5, 13))
        T = min(_size(rng, 1, 32768), max(1, 260_000_000 // (P * D * N)))
    state = direction == "forward" and rng.random() < 0.6
    S, ragged = rng.choice((1, 1, 2, 4, T, _size(rng, 1, 64))), rng.random() < 0.4
    if not ragged:
        S = min(S, T)
        T = T // S * S
    S = min(S, 4096)
    if not ragged and T % S:
        T = max(S, T // S * S)
    if op == "conv":
        c = _conv("", direction, P, T, S, D, rng.choice((4, 4, 3, 2)), act, rng.random() < 0.8, ragged, state)
    else:
        if state:       # the states are no more than the rows' work
            S = max(1, min(S, 16_000_000 // (P * D * N)))
            T = T if ragged else max(1, T // S) * S
        c = _scan("", direction, P, T, S, D, N, act, rng.random() < 0.7, ragged, state)
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, shift=0.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(shift, scale, generator=gen).to(dtype)

    c = case
    s = {"case": dict(c)}
    P = c["P"]
    if c["op"] == "ortho":
        # a gradient has a few large directions and many small ones
        m, n = c["m"], c["n"]
        r = max(1, min(m, n) // 4)
        g = normal(P, m, r) @ normal(P, r, n) * (1e-3 / math.sqrt(r)) + normal(P, m, n, scale=3e-4)
        s["grad"] = g.to(TYPES[c["grad"]])
        if c["momentum"]:
            s["momentum"] = g * 7.0 + normal(P, m, n, scale=2e-3)
        s["out"] = torch.empty((P, m, n), dtype=torch.bfloat16, device="cuda")
        return s
    T, S, D, A = c["T"], c["S"], c["D"], TYPES[c["act"]]
    s["starts"] = None
    if c["ragged"]:
        # S sequences of any length, none and one among them, behind a few unused rows and before a few more
        cut = torch.rand((P, S + 1), generator=gen, device="cuda", dtype=torch.float64)
        lo, hi = min(3, T // 8), T - T // 50
        cut = (lo + cut * (hi - lo + 1)).long().clamp_(lo, hi).sort(1)[0]
        cut[:, 0] = lo
        s["starts"] = cut.int()
    rows = lambda scale=1.0, shift=0.0: normal(P, T, D, dtype=A, scale=scale, shift=shift)  # noqa: E731
    s["x"] = rows(0.7)
    s["out"] = torch.zeros((P, T, D), dtype=A, device="cuda")
    if c["op"] == "conv":
        s["w"], s["bias"] = normal(P, D, c["W"], scale=c["W"] ** -0.5), normal(P, D, scale=0.1)
        if c["state"]:
            s["state"] = normal(P, S, c["W"] - 1, D, dtype=A, scale=0.7)
        if c["dir"] == "training":
            s["d_out"] = rows(1e-2)
            s["dx"], s["dw"], s["d_bias"] = torch.zeros_like(s["x"]), torch.empty_like(s["w"]), torch.empty_like(s["bias"])
        return s
    # time steps of 0.001 to 0.1 before the tokens move them, decays of 1 to N, as such models begin
    N = c["N"]
    step = torch.exp(torch.empty((P, D), device="cuda").uniform_(math.log(1e-3), math.log(1e-1), generator=gen))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["dt"] = rows(0.5)
    s["a_log"] = torch.log(torch.arange(1, N + 1, device="cuda", dtype=torch.float32)).expand(P, D, N) + normal(P, D, N, scale=0.1)
    s["b"], s["c"] = normal(P, T, N, dtype=A), normal(P, T, N, dtype=A)
    s["skip"] = normal(P, D, scale=0.1, shift=1.0)
    if c["gate"]:
        s["z"] = rows()
    if c["state"]:
        s["state"] = normal(P, S, D, N, scale=0.3)
    if c["dir"] == "training":
        s["d_out"] = rows(1e-2)
        for k in ("x", "dt", "b", "c") + (("z",) if c["gate"] else ()):
            s["d_" + k] = torch.zeros_like(s[k])
        for k in ("a_log", "skip", "dt_bias"):
            s["d_" + k] = torch.empty_like(s[k])
    return s


# ------------------------------------------------------------------------------------------------ plain form
def _sequences(s):
    """(sequence of every row, its start, its length, whether the row belongs to one), each [P, T]."""
    c = s["case"]
    P, T, S = c["P"], c["T"], c["S"]
    starts = s["starts"]
    if starts is None:
        starts = (torch.arange(S + 1, device="cuda") * (T // S)).expand(P, S + 1)
    starts = starts.long().contiguous()
    t = torch.arange(T, device="cuda").expand(P, T).contiguous()
    seq = torch.searchsorted(starts, t, right=True) - 1
    live = (seq >= 0) & (seq < S)
    seq = seq.clamp(0, S - 1)
    begin = starts.gather(1, seq)
    return starts, seq, begin, live


def _conv_plain(s):
    c = s["case"]
    P, T, S, D, W = (c[k] for k in "PTSDW")
    starts, seq, begin, live = _sequences(s)
    x = s["x"].float()
    old = s["state"].float() if c["state"] else torch.zeros((P, S, max(W - 1, 1), D), device="cuda")
    who = torch.arange(P, device="cuda")[:, None]
    t = torch.arange(T, device="cuda").expand(P, T)

    def before(k):          # the input k tokens before every row's, of its sequence or of the state
        at = t - begin - k
        inside = x[who, (t - k).clamp(min=0)]
        return inside if W == 1 else torch.where((at >= 0)[..., None], inside, old[who, seq, (at + W - 1).clamp(0, max(W - 2, 0))])

    taps = [before(W - 1 - j) for j in range(W)]
    pre = sum(tap * s["w"][:, None, :, j] for j, tap in enumerate(taps)) + s["bias"][:, None]
    gate = 1 / (1 + torch.exp(-pre))
    got = {"out": s["out"].copy_(torch.where(live[..., None], pre * gate if c["silu"] else pre, s["out"].float()))}
    if c["state"]:
        length = starts[:, 1:] - starts[:, :-1]
        at = length[..., None] + torch.arange(W - 1, device="cuda")           # of the old state with the sequence behind it
        row = (starts[:, :-1, None] + at - (W - 1)).clamp(0, T - 1)
        kept = old[who[..., None], torch.arange(S, device="cuda")[:, None], at.clamp(max=W - 2)]
        s["state"].copy_(torch.where((at >= W - 1)[..., None], x[who[..., None], row], kept))
        got["state"] = s["state"]
    if c["dir"] == "training":
        d = s["d_out"].float() * (gate * (1 + pre * (1 - gate)) if c["silu"] else 1.0)
        d = torch.where(live[..., None], d, 0.0)
        got["dw"], got["d_bias"] = torch.stack([(d * tap).sum(1) for tap in taps], -1), d.sum(1)
        dx = torch.zeros_like(x)
        for k in range(W):
            reach = torch.where(((t - begin - k) >= 0)[..., None], d, 0.0)
            dx[:, :T - k] += reach[:, k:] * s["w"][:, None, :, W - 1 - k]
        got["dx"] = dx.to(s["x"].dtype)
    return got


def _recur(a, b):
    """h_t = a_t h_(t-1) + b_t over dimension 1, by doubling; a and b are overwritten."""
    k, T = 1, a.shape[1]
    while k < T:
        b[:, k:] += a[:, k:] * b[:, :-k]
        a[:, k:] = a[:, k:] * a[:, :-k]
        k *= 2
    return b


def _scan_plain(s):
    c = s["case"]
    P, T, S = c["P"], c["T"], c["S"]
    starts, seq, begin, live = _sequences(s)
    t = torch.arange(T, device="cuda").expand(P, T)
    first, live = (t == begin) & live, live[..., None]
    who = torch.arange(P, device="cuda")[:, None]
    x, z = s["x"].float(), s["z"].float() if c["gate"] else None
    pre = s["dt"].float() + s["dt_bias"][:, None]
    e = torch.exp(-pre.abs())
    delta = torch.where(live, pre.clamp(min=0) + torch.log1p(e), 0.0)
    A = -torch.exp(s["a_log"])[:, None]
    B, C = s["b"].float()[:, :, None], s["c"].float()[:, :, None]
    a = torch.exp(delta[..., None] * A)
    h = (delta * torch.where(live, x, 0.0))[..., None] * B
    if c["state"]:
        h += torch.where(first[..., None, None], a * s["state"][who, seq], 0.0)
    cut = torch.where(first[..., None, None], 0.0, a)
    keep = cut.clone() if c["dir"] == "training" else None
    h = _recur(cut, h)
    y = (h * C).sum(-1) + s["skip"][:, None] * x
    sig = 1 / (1 + torch.exp(-z)) if c["gate"] else None
    out = y * z * sig if c["gate"] else y
    got = {"out": s["out"].copy_(torch.where(live, out, s["out"].float()))}
    if c["state"]:
        length = starts[:, 1:] - starts[:, :-1]
        last = h[who, (starts[:, 1:] - 1).clamp(min=0)]
        s["state"].copy_(torch.where((length > 0)[..., None, None], last, s["state"]))
        got["state"] = s["state"]
    if c["dir"] == "forward":
        return got
    d = torch.where(live, s["d_out"].float(), 0.0)
    if c["gate"]:
        got["d_z"] = (d * y * (sig * (1 + z * (1 - sig)))).to(s["z"].dtype)
        d = d * z * sig
    got["d_skip"] = (d * x).sum(1)
    # the adjoint runs backwards, through the decay of the next row
    back = torch.zeros_like(keep)
    back[:, :-1] = keep[:, 1:]
    g = _recur(back.flip(1), (d[..., None] * C).flip(1)).flip(1)
    del back
    got["d_c"] = (h * d[..., None]).sum(2).to(s["c"].dtype)
    got["d_b"] = (g * (delta * x)[..., None]).sum(2).to(s["b"].dtype)
    du = (g * B).sum(-1)
    h[:, 1:] = h[:, :-1].clone()
    h[:, 0] = 0
    h *= keep
    h *= g                                       # g a h_(t-1)
    got["d_a_log"] = (h * delta[..., None]).sum(1) * A[:, 0]
    ddelta = (h * A).sum(-1) + du * x
    got["d_x"] = torch.where(live, delta * du + s["skip"][:, None] * d, 0.0).to(s["x"].dtype)
    ddt = torch.where(live, ddelta * torch.where(pre >= 0, 1 / (1 + e), e / (1 + e)), 0.0)
    got["d_dt"], got["d_dt_bias"] = ddt.to(s["dt"].dtype), ddt.sum(1)
    return got


def _ortho_plain(s):
    c, got = s["case"], {}
    U = s["grad"].float()
    if c["momentum"]:
        m = s["momentum"].mul_(MU).add_(U)
        U, got["momentum"] = U + MU * m, m
    X = U / (U.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    if c["m"] > c["n"]:
        X = X.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        G = X @ X.transpose(1, 2)
        X = COEF[0] * X + (COEF[1] * G + COEF[2] * (G @ G)) @ X
    if c["m"] > c["n"]:
        X = X.transpose(1, 2)
    got["out"] = X.to(torch.bfloat16)
    return got


# ------------------------------------------------------------------------------------------------ the repository's kernels
def _own_op(s):
    """The bound operator that a user's program keeps beside its buffers: made at the first pass."""
    from paper_1905_10395_b200 import lm
    c = s["case"]
    if c["op"] == "ortho":
        return lm.Orthogonalize(s["grad"], s["out"], momentum=s.get("momentum"), mu=MU, nesterov=True, steps=STEPS,
                                coefficients=COEF, eps=EPS)
    where = {"sequences": c["S"]} if s["starts"] is None else {"starts": s["starts"]}
    grads = c["dir"] == "training"
    if c["op"] == "conv":
        names = ("bias", "out", "state") + (("d_out", "dx", "dw", "d_bias") if grads else ())
        return lm.CausalConv(s["x"], s["w"], act="silu" if c["silu"] else "identity", **{k: s[k] for k in names if k in s}, **where)
    names = ("z", "skip", "dt_bias", "out", "state")
    if grads:
        names += ("d_out", "d_x", "d_dt", "d_a_log", "d_b", "d_c", "d_z", "d_skip", "d_dt_bias")
    return lm.SelectiveScan(s["x"], s["dt"], s["a_log"], s["b"], s["c"], **{k: s[k] for k in names if k in s}, **where)


def _run_own(s):
    c = s["case"]
    if "op" not in s:
        s["op"] = _own_op(s)
    s["op"].forward()
    if c["op"] == "ortho":
        return {k: s[k] for k in ("out", "momentum") if k in s}
    if c["dir"] == "training":
        s["op"].backward()
    names = ("out", "state", "dx", "dw", "d_bias", "d_x", "d_dt", "d_a_log", "d_b", "d_c", "d_z", "d_skip", "d_dt_bias")
    return {k: s[k] for k in names if k in s}


def run(state):
    if own:
        return _run_own(state)
    return {"conv": _conv_plain, "scan": _scan_plain, "ortho": _ortho_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "ortho":
        P, least, most = c["P"], min(c["m"], c["n"]), max(c["m"], c["n"])
        each = BYTES[c["grad"]] + 2 + (8 if c["momentum"] else 0)
        # a step: half of X X^T and half of G G (both are symmetric), and the product with X
        return {"bytes": P * least * most * each, "flops": P * STEPS * (3.0 * least * least * most + 1.0 * least ** 3)}
    P, S, D, a = c["P"], c["S"], c["D"], BYTES[c["act"]]
    n = P * (c["T"] - (c["T"] // 50 + min(3, c["T"] // 8) if c["ragged"] else 0))
    training = c["dir"] == "training"
    if c["op"] == "conv":
        vectors = P * D * 4 * (c["W"] + 1) * (3 if training else 1)
        state = 2 * P * S * (c["W"] - 1) * D * a if c["state"] else 0
        return {"bytes": n * D * a * (5 if training else 2) + vectors + state, "flops": n * D * (2 * c["W"] + 6) * (4 if training else 1)}
    N, rows = c["N"], 4 if c["gate"] else 3
    vectors = P * D * 4 * (N + 2) * (3 if training else 1)
    state = 8 * P * S * D * N if c["state"] else 0
    # forward: x, dt, z -> out; gradient: x, dt, z, d_out -> dx, d_dt, dz
    bytes_ = n * a * (D * (rows + (2 * rows - 1 if training else 0)) + N * (6 if training else 2)) + vectors + state
    return {"bytes": bytes_, "flops": n * D * N * (22 if training else 6)}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = case
    f = lambda k: s[k].to(torch.float64)  # noqa: E731
    P = c["P"]
    if c["op"] == "ortho":
        # with the singular values: a step maps each to a v + b v^3 + c v^5
        got = {}
        U = f("grad")
        if c["momentum"]:
            got["momentum"] = MU * f("momentum") + U
            U = U + MU * got["momentum"]
        tall = c["m"] > c["n"]
        U = U.mT if tall else U
        X = U / (torch.linalg.matrix_norm(U)[:, None, None] + EPS)
        # X = Q v R, so p(X) = Q p(v) / v Q^T X; the eigenvectors of X X^T are Q
        v2, Q = torch.linalg.eigh(X @ X.mT)
        v2 = v2.clamp(min=0)
        factor = torch.ones_like(v2)
        for _ in range(STEPS):
            w = v2 * factor * factor
            factor = factor * (COEF[0] + COEF[1] * w + COEF[2] * w * w)
        X = (Q * factor.unsqueeze(1)) @ (Q.mT @ X)
        got["out"] = X.mT if tall else X
        return got
    T, S, D = c["T"], c["S"], c["D"]
    edges = s["starts"].tolist() if c["ragged"] else [[i * (T // S) for i in range(S + 1)]] * P
    training = c["dir"] == "training"
    if c["op"] == "conv":
        W = c["W"]
        got = {"out": f("out")}
        if c["state"]:
            got["state"] = f("state")
        if training:
            got |= {"dx": torch.zeros_like(f("x")), "dw": torch.zeros_like(f("w")), "d_bias": torch.zeros_like(f("bias"))}
        if P * S > 600:
            return None
        for p in range(P):
            w, bias = f("w")[p], f("bias")[p]
            for i, (lo, hi) in enumerate(zip(edges[p], edges[p][1:])):
                old = got["state"][p, i] if c["state"] else torch.zeros((W - 1, D), dtype=torch.float64, device="cuda")
                v = torch.cat([old, s["x"][p, lo:hi].double()])
                if c["state"]:
                    got["state"][p, i] = v[hi - lo:]
                if hi == lo:
                    continue
                u = v.T.unsqueeze(0)                    # [1, D, W - 1 + length]
                wide = u.unfold(2, W, 1)[0]             # [D, length, W]
                pre = (wide * w[:, None]).sum(-1) + bias[:, None]
                sg = torch.sigmoid(pre)
                got["out"][p, lo:hi] = (pre * sg if c["silu"] else pre).T
                if training:
                    d = s["d_out"][p, lo:hi].double().T * (sg + pre * sg * (1 - sg) if c["silu"] else 1.0)
                    got["dw"][p] += torch.einsum("dt,dtw->dw", d, wide)
                    got["d_bias"][p] += d.sum(1)
                    back = torch.nn.functional.pad(d, (0, W - 1)).unfold(1, W, 1)       # d of the next W rows
                    got["dx"][p, lo:hi] = (back * w.flip(1)[:, None]).sum(-1).T
        return got
    # scan: the recurrence token by token, forwards and backwards
    N = c["N"]
    if T * (3 if training else 1) > 110_000:
        return None
    first = torch.zeros((T, P), dtype=torch.long) - 1
    live = torch.zeros((T, P), dtype=torch.bool)
    ends = torch.zeros((T, P), dtype=torch.long) - 1
    for p in range(P):
        live[edges[p][0]:edges[p][-1], p] = True
        for i, (lo, hi) in enumerate(zip(edges[p], edges[p][1:])):
            if hi > lo:
                first[lo, p], ends[hi - 1, p] = i, i
    has_first, has_end = [bool(v) for v in (first >= 0).any(1)], [bool(v) for v in (ends >= 0).any(1)]
    first, ends, live = first.cuda(), ends.cuda(), live.cuda()
    A = -torch.exp(f("a_log"))
    got = {"out": f("out")}
    state = f("state") if c["state"] else None
    pre = f("dt") + f("dt_bias")[:, None]
    delta = torch.nn.functional.softplus(pre, threshold=60.0) * live.T[..., None]
    u = delta * f("x")
    h = torch.zeros((P, D, N), dtype=torch.float64, device="cuda")
    hs = torch.empty((T, P, D, N), dtype=torch.float64, device="cuda") if training else None
    y = torch.empty((P, T, D), dtype=torch.float64, device="cuda")
    B, C = f("b"), f("c")
    new = state.clone() if c["state"] else None
    who = torch.arange(P, device="cuda")
    for t in range(T):
        if has_first[t]:
            fresh = state[who, first[t].clamp(min=0)] if c["state"] else 0.0
            h = torch.where((first[t] >= 0)[:, None, None], fresh, h)
        h = torch.exp(delta[:, t, :, None] * A).mul_(h).addcmul_(u[:, t, :, None], B[:, t, None])
        y[:, t] = torch.bmm(h, C[:, t, :, None])[..., 0]
        if training:
            hs[t] = h
        if c["state"] and has_end[t]:
            hit = ends[t] >= 0
            new[who[hit], ends[t][hit]] = h[hit]
    y += f("skip")[:, None] * f("x")
    sg = torch.sigmoid(f("z")) if c["gate"] else 1.0
    gate = f("z") * sg if c["gate"] else 1.0
    got["out"] = torch.where(live.T[..., None], y * gate, got["out"])
    if c["state"]:
        got["state"] = new
    if not training:
        return got
    mask = live.T[..., None].double()
    d = f("d_out") * mask
    if c["gate"]:
        got["d_z"] = d * y * (sg + gate * (1 - sg))
    d = d * gate
    got["d_skip"] = (d * f("x")).sum(1)
    names = {"d_b": B, "d_c": C, "d_x": u, "d_dt": u}
    got |= {k: torch.zeros_like(v) for k, v in names.items()}
    dA = torch.zeros_like(A)
    zero = torch.zeros_like(h)
    carry = zero                                            # what reaches h_t from the rows behind t
    xs = f("x")
    for t in reversed(range(T)):
        g = torch.addcmul(carry, d[:, t, :, None], C[:, t, None])
        got["d_c"][:, t] = torch.bmm(d[:, t, None], hs[t])[:, 0]
        got["d_b"][:, t] = torch.bmm(u[:, t, None], g)[:, 0]
        gb = torch.bmm(g, B[:, t, :, None])[..., 0]
        carry = torch.exp(delta[:, t, :, None] * A).mul_(g)
        if has_first[t]:
            carry = torch.where((first[t] >= 0)[:, None, None], 0.0, carry)
        q = carry * hs[t - 1] if t else zero
        dA.addcmul_(q, delta[:, t, :, None])
        got["d_x"][:, t] = gb * delta[:, t]
        got["d_dt"][:, t] = gb * xs[:, t] + (q * A).sum(-1)
    got["d_x"] = (got["d_x"] + f("skip")[:, None] * d) * mask
    got["d_dt"] = got["d_dt"] * torch.sigmoid(pre) * mask
    got["d_dt_bias"] = got["d_dt"].sum(1)
    got["d_a_log"] = dA * A
    return got
