"""Plain 64-bit restatements of the convolution, the scan and the orthogonalisation (include/lsgd.h), on the CPU, token by token.

Beside a result stands the sum of the magnitudes that it is made of: what a bound on its rounding errors is relative to."""
import torch

F64 = torch.float64


def edges_of(P, T, S, starts):
    """Rows at which every worker's sequences begin, and the end of all: P lists of S + 1."""
    if starts is None:
        return [[i * (T // S) for i in range(S + 1)]] * P
    s = starts if starts.dim() == 2 else starts.expand(P, -1)
    return [[min(max(int(v), 0), T) for v in row] for row in s]


# ---- convolution
def conv(x, w, bias=None, state=None, d_out=None, edges=None, act="silu"):
    """x float64 [P, T, D], w [P, D, W], bias [P, D], state [P, S, W - 1, D]: ({name: value}, {name: magnitudes}).  Rows of no sequence
    are NaN in the results."""
    P, T, D = x.shape
    W = w.shape[2]
    nan = torch.full_like(x, float("nan"))
    got, size = {"out": nan.clone()}, {"out": nan.clone()}
    if state is not None:
        got["state"] = state.clone()
    if d_out is not None:
        for b in (got, size):
            b["dx"], b["dw"], b["d_bias"] = nan.clone(), torch.zeros_like(w), torch.zeros((P, D), dtype=F64)
    for p in range(P):
        for i, (lo, hi) in enumerate(zip(edges[p], edges[p][1:])):
            n = hi - lo
            if n <= 0:
                continue
            old = torch.zeros((W - 1, D), dtype=F64) if state is None else state[p, i]
            v = torch.cat([old, x[p, lo:hi]])
            taps = [v[j:j + n] for j in range(W)]
            pre, mag = torch.zeros((n, D), dtype=F64), torch.zeros((n, D), dtype=F64)
            for j in range(W):
                pre, mag = pre + w[p, :, j] * taps[j], mag + (w[p, :, j] * taps[j]).abs()
            if bias is not None:
                pre, mag = pre + bias[p], mag + bias[p].abs()
            sg = torch.sigmoid(pre)
            got["out"][p, lo:hi] = pre * sg if act == "silu" else pre
            # |act'| <= 1.1
            size["out"][p, lo:hi] = 1.1 * mag
            if state is not None:
                got["state"][p, i] = v[n:]
            if d_out is None:
                continue
            slope = sg * (1 + pre * (1 - sg)) if act == "silu" else torch.ones_like(pre)
            g = d_out[p, lo:hi] * slope
            # |act''| <= 0.5: the slope is off by what pre is off
            gm = d_out[p, lo:hi].abs() * ((sg * (1 + pre.abs() * (1 - sg)) + 0.5 * mag) if act == "silu" else 1.0)
            for j in range(W):
                got["dw"][p, :, j] += (g * taps[j]).sum(0)
                size["dw"][p, :, j] += (gm * taps[j].abs()).sum(0)
            got["d_bias"][p] += g.sum(0)
            size["d_bias"][p] += gm.sum(0)
            for b, q, ww in ((got, g, w[p]), (size, gm, w[p].abs())):
                dx = torch.zeros((n, D), dtype=F64)
                for k in range(min(W, n)):
                    dx[:n - k] += q[k:] * ww[:, W - 1 - k]
                b["dx"][p, lo:hi] = dx
    return got, size


# ---- scan
def scan(x, dt, a_log, b, c, z=None, skip=None, dt_bias=None, state=None, d_out=None, edges=None):
    """float64: ({name: value}, {name: magnitudes}).  Rows of no sequence are NaN in the results."""
    P, T, D = x.shape
    N = a_log.shape[2]
    nan = torch.full_like(x, float("nan"))
    got, size = {"out": nan.clone()}, {"out": nan.clone()}
    if state is not None:
        got["state"], size["state"] = state.clone(), state.abs()
    if d_out is not None:
        for q in (got, size):
            q["d_x"], q["d_dt"], q["d_a_log"] = nan.clone(), nan.clone(), torch.zeros_like(a_log)
            q["d_b"], q["d_c"] = torch.full_like(b, float("nan")), torch.full_like(c, float("nan"))
            q["d_skip"], q["d_dt_bias"] = torch.zeros((P, D), dtype=F64), torch.zeros((P, D), dtype=F64)
            q["d_z"] = nan.clone()
    for p in range(P):
        A = -torch.exp(a_log[p])
        sk = torch.zeros(D, dtype=F64) if skip is None else skip[p]
        for i, (lo, hi) in enumerate(zip(edges[p], edges[p][1:])):
            if hi <= lo:
                continue
            pre = dt[p, lo:hi] + (0 if dt_bias is None else dt_bias[p])
            delta = torch.nn.functional.softplus(pre, threshold=80.0)
            xs, B, C = x[p, lo:hi], b[p, lo:hi], c[p, lo:hi]
            a = torch.exp(delta[..., None] * A)
            u = (delta * xs)[..., None] * B[:, None]
            h = torch.zeros((D, N), dtype=F64) if state is None else state[p, i].clone()
            m = h.abs()
            hs, ms = [], []
            for t in range(hi - lo):
                h, m = a[t] * h + u[t], a[t] * m + u[t].abs()
                hs.append(h)
                ms.append(m)
            if state is not None:
                got["state"][p, i], size["state"][p, i] = h, m
            hs, ms = torch.stack(hs), torch.stack(ms)
            y, ym = (hs * C[:, None]).sum(-1) + sk * xs, (ms * C[:, None].abs()).sum(-1) + (sk * xs).abs()
            zz = torch.ones_like(xs) if z is None else z[p, lo:hi]
            sg = torch.sigmoid(zz)
            gate = torch.ones_like(xs) if z is None else zz * sg
            got["out"][p, lo:hi], size["out"][p, lo:hi] = y * gate, ym * gate.abs()
            if d_out is None:
                continue
            up = d_out[p, lo:hi]
            got["d_z"][p, lo:hi] = up * y * sg * (1 + zz * (1 - sg))
            size["d_z"][p, lo:hi] = up.abs() * ym * sg * (1 + zz.abs() * (1 - sg))
            d = up * gate
            carry, cm = torch.zeros((D, N), dtype=F64), torch.zeros((D, N), dtype=F64)
            slope = torch.sigmoid(pre)
            for t in reversed(range(hi - lo)):
                g, gm = d[t][:, None] * C[t] + carry, (d[t][:, None] * C[t]).abs() + cm
                for q, gg, hh, dd, uu, BB in ((got, g, hs[t], d[t], (delta * xs)[t], B[t]),
                                              (size, gm, ms[t], d[t].abs(), (delta * xs)[t].abs(), B[t].abs())):
                    q["d_c"][p, lo + t] = (dd[:, None] * hh).sum(0)
                    q["d_b"][p, lo + t] = (gg * uu[:, None]).sum(0)
                carry, cm = a[t] * g, a[t] * gm
                prev, pm = (hs[t - 1], ms[t - 1]) if t else (torch.zeros_like(h), torch.zeros_like(h))
                q, qm = carry * prev, cm * pm
                gb, gbm = (g * B[t]).sum(-1), (gm * B[t].abs()).sum(-1)
                got["d_a_log"][p] += q * delta[t][:, None] * A
                size["d_a_log"][p] += qm * delta[t][:, None] * A.abs()
                got["d_x"][p, lo + t] = delta[t] * gb + sk * d[t]
                size["d_x"][p, lo + t] = delta[t] * gbm + (sk * d[t]).abs()
                got["d_dt"][p, lo + t] = (xs[t] * gb + (q * A).sum(-1)) * slope[t]
                size["d_dt"][p, lo + t] = (xs[t].abs() * gbm + (qm * A.abs()).sum(-1)) * slope[t]
            got["d_skip"][p] += (d * xs).sum(0)
            size["d_skip"][p] += (d * xs).abs().sum(0)
            got["d_dt_bias"][p] += got["d_dt"][p, lo:hi].sum(0)
            size["d_dt_bias"][p] += size["d_dt"][p, lo:hi].sum(0)
    return got, size


# ---- orthogonalisation
def ortho(grad, momentum=None, mu=0.95, nesterov=True, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0):
    """float64 [P, m, n]: (out, momentum)."""
    U = grad
    if momentum is not None:
        momentum = mu * momentum + grad
        U = grad + mu * momentum if nesterov else momentum
    X = U / (U.square().sum((1, 2), keepdim=True).sqrt() + eps)
    a, b, c = coefficients
    tall = X.shape[1] > X.shape[2]
    X = X.mT if tall else X
    for _ in range(steps):
        G = X @ X.mT
        X = a * X + (b * G + c * G @ G) @ X
    return scale * (X.mT if tall else X), momentum
