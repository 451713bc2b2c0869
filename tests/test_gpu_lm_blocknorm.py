"""GPU check of the block-boundary norms (lsgd_blocknorm_*) against their 64-bit restatement: every type, mode and kind of
row, odd sizes, strides, shared and broadcast operands, in-place use, and the gradient against differences.

Bounds.  An fp32 result of k roundings is within k 2^-24 of the sum of the magnitudes that it is made of.  A row sum of D
values is a tree (16 serial additions, 5 + 4 levels), so 1 / sqrt(..) is within 2^-19; the other factors add less: 2^-18 of
the magnitudes, plus half a unit (2^-9 of the value) where a result is stored in bf16.  Gradients subtract the row's mean
term, so their magnitude is that of both terms.  Sums over T <= 300 rows add at most 300 2^-24 < 2^-15 of the terms."""
import itertools

import pytest
import torch

from tests import _lm_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, torch.float32), "mixed": (torch.float32, torch.bfloat16), "bf16": (torch.bfloat16, torch.bfloat16)}
REL = 2.0 ** -18


def _close(name, got, want, size, stored, rel=REL):
    got = got.double().cpu()
    half = 2.0 ** -8 if stored == torch.bfloat16 else 0.0
    bound = rel * size + half * want.abs() + 1e-35
    bad = (got - want).abs() > bound
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {((got - want).abs() / bound).max():.3g} of the bound"
    assert torch.isfinite(got).all()


def _draw(gen, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale + shift).to(dtype)


def _strides(kind, P, T, D):
    return {"rows": (T * D, D, 1), "padded": (T * (D + 5) + 3, D + 5, 1), "aligned": (T * ((D + 15) // 8 * 8), (D + 15) // 8 * 8, 1),
            "interleaved": (D, P * D, 1)}[kind]


def run(P, T, D, types, y=True, post=True, pre=True, gate="none", act="identity", kind="rows", offset=0, seed=0, alpha=0.9,
        beta=0.7, eps=1e-5, zero_row=False, accumulate=False, in_place=False, has_d_out=True, scale=1.0):
    from paper_1905_10395_b200 import lm
    R, A = TYPES[types]
    gen = torch.Generator().manual_seed(seed)
    host = {"x": _draw(gen, (P, T, D), R, 2.0 * scale)}
    if y:
        host["y"] = _draw(gen, (P, T, D), A, scale)
        if zero_row and T:
            host["y"][:, T // 2] = 0
    if zero_row and T:
        host["x"][:, T // 2] = 0
    if gate == "channel":
        host["gate"] = _draw(gen, (P, D), torch.float32, 1.0)
    elif gate == "token":
        host["gate"] = _draw(gen, (P, T, D), A, 1.0)
    if y and post:
        host["w_post"] = _draw(gen, (P, D), torch.float32, 0.3, 1.0)
    if pre:
        host["w_pre"] = _draw(gen, (P, D), torch.float32, 0.3, 1.0)
    strides = _strides(kind, P, T, D)

    def rows(dtype, fill=None):
        return ref.Guarded((P, T, D), strides, dtype, offset, fill)

    dev = {k: (rows(v.dtype, v) if v.dim() == 3 else ref.Guarded((P, D), (D + 3, 1), v.dtype, 1, v)) for k, v in host.items()}
    f64 = {k: v.double() for k, v in host.items()}
    opt = dict(act=act, alpha=alpha, beta=beta, eps=eps)
    view = lambda k: dev[k].view if k in dev else None  # noqa: E731

    # forward
    out = (dev["x"] if in_place else rows(R)) if y else None
    h = rows(A) if pre else None
    op = lm.BlockNorm(x=view("x"), y=view("y"), gate=view("gate"), w_post=view("w_post"), w_pre=view("w_pre"),
                      out=out.view if out else None, h=h.view if h else None, post_norm=post, gate_act=act, alpha=alpha, beta=beta,
                      eps=eps)
    op.forward()
    torch.cuda.synchronize()
    want_out, want_h = ref.blocknorm_forward(f64["x"], f64.get("y"), f64.get("gate"), f64.get("w_post"), f64.get("w_pre"), **opt)
    size = f64["x"].abs() * abs(alpha)
    if y:
        size = size + (want_out - alpha * f64["x"]).abs()
        _close("out", out.view, want_out, size, R)
    else:
        size = f64["x"].abs()
    if pre:
        r = 1 / torch.sqrt(want_out.square().mean(-1, keepdim=True) + eps)
        _close("h", h.view, want_h, size * r * f64["w_pre"][:, None].abs(), A)
        _close("rstd_pre", op.rstd_pre, r[..., 0], 4 * r[..., 0], torch.float32)
    if y and post:
        r = 1 / torch.sqrt(f64["y"].square().mean(-1) + eps)
        _close("rstd_post", op.rstd_post, r, r, torch.float32)
    for g in list(dev.values()) + [b for b in (out, h) if b]:
        assert g.intact()

    # backward, from x' as stored
    stored = (out.view if y else dev["x"].view).cpu().clone()
    d_out = rows(R, _draw(gen, (P, T, D), R, 1.0)) if has_d_out else None
    d_h = rows(A, _draw(gen, (P, T, D), A, 1.0)) if pre else None
    start = {}
    res = {"dx": d_out if in_place and has_d_out else rows(R)}
    d_out_host = d_out.view.cpu().double() if d_out else None
    if y:
        res["dy"] = rows(A)
    if gate == "token":
        res["d_gate"] = rows(A)
    vectors = (["d_gate"] if gate == "channel" else []) + (["dw_post"] if y and post else []) + (["dw_pre"] if pre else [])
    for k in vectors:
        start[k] = _draw(gen, (P, D), torch.float32)
        res[k] = ref.Guarded((P, D), (D + 1, 1), torch.float32, 0, start[k])
    op2 = lm.BlockNorm(y=view("y"), gate=view("gate"), w_post=view("w_post"), w_pre=view("w_pre"),
                       out=out.view if y else dev["x"].view, rstd_post=op.rstd_post, rstd_pre=op.rstd_pre,
                       d_out=d_out.view if d_out else None, d_h=d_h.view if d_h else None, post_norm=post, gate_act=act,
                       alpha=alpha, beta=beta, eps=eps, accumulate=accumulate, **{k: v.view for k, v in res.items()})
    op2.backward()
    torch.cuda.synchronize()
    want, terms = ref.blocknorm_backward(d_out_host, d_h.view.cpu().double() if d_h else None, stored.double(), f64.get("y"),
                                         f64.get("gate"), f64.get("w_post"), f64.get("w_pre"), **opt)
    # x' is stored in R and 1 / sqrt(..) was taken of it before that rounding
    lost = 2.0 ** -8 if R == torch.bfloat16 else 0.0
    up = torch.zeros(P, T, D, dtype=torch.float64)
    if pre:
        r = 1 / torch.sqrt(stored.double().square().mean(-1, keepdim=True) + eps)
        n = stored.double() * r
        up = (d_h.view.cpu().double() * f64["w_pre"][:, None])
        size = r * (up.abs() + n.abs() * (up * n).abs().mean(-1, keepdim=True))
    else:
        size = torch.zeros_like(up)
    if d_out is not None:
        size = size + d_out_host.abs()
    _close("dx", res["dx"].view, want["dx"], size * (abs(alpha) if y else 1.0), R, REL + lost)
    if y:
        a = ref.gate_act(f64["gate"] if gate == "token" else f64["gate"][:, None], act) if gate != "none" else torch.ones(1, dtype=torch.float64)
        s = size * abs(beta) * a.abs()
        if post:
            ry = 1 / torch.sqrt(f64["y"].square().mean(-1, keepdim=True) + eps)
            ny = f64["y"] * ry
            s = s * f64["w_post"][:, None].abs()
            s = ry * (s + ny.abs() * (s * ny.abs()).mean(-1, keepdim=True))
        _close("dy", res["dy"].view, want["dy"], s + 0 * want["dy"], A, 4 * REL + lost)
        if gate == "token":
            u = f64["y"] if not post else ny * f64["w_post"][:, None]
            _close("d_gate", res["d_gate"].view, want["d_gate"], size * abs(beta) * u.abs(), A, 4 * REL + lost)
    # a sum's own terms differ from the formula's by the error of g: bounded through the sum of |terms of g| * |factors|
    for k in vectors:
        base = start[k].double() if accumulate else 0.0
        if k == "dw_pre":
            size_k = terms[k]
        else:
            u = f64["y"] if not post else ny
            if k == "d_gate" and post:
                u = u * f64["w_post"][:, None]
            factor = u.abs() if k == "d_gate" else u.abs() * a.abs()
            size_k = (size * abs(beta) * factor).sum(1)
        total = want[k] + base
        _close(k, res[k].view, total, size_k + (start[k].double().abs() if accumulate else 0.0), torch.float32, 2.0 ** -15 + lost)
    for g in list(dev.values()) + list(res.values()) + [b for b in (out, h, d_out, d_h) if b]:
        assert g.intact()
    return op, op2


MODES = [dict(y=False), dict(post=False), dict(post=False, pre=False), dict(pre=False), dict(), dict(gate="channel", act="sigmoid"),
         dict(gate="channel", act="tanh", post=False), dict(gate="channel", pre=False), dict(gate="token", act="sigmoid"),
         dict(gate="token", act="tanh", pre=False), dict(gate="token", post=False), dict(gate="token", post=False, pre=False),
         dict(has_d_out=False)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("mode", range(len(MODES)))
def test_every_mode_and_type(mode, types):
    run(2, 19, 136, types, seed=mode, **MODES[mode])          # ragged: 136 values are not 16 for each of 16 threads
    run(2, 19, 256, types, seed=mode, **MODES[mode])          # whole: 16 threads of 16 values
    run(1, 13, 133, types, seed=mode, **MODES[mode])          # rows off 16-byte boundaries
    run(2, 5, 67, types, seed=mode, kind="padded", offset=1, **MODES[mode])   # one value at a time


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("D", [1, 2, 3, 7, 8, 9, 15, 16, 17, 63, 64, 65, 255, 256, 257, 511, 512, 513, 1001, 1024, 1500, 2048, 2055,
                               4095, 4096, 4097, 4507, 8176, 8185, 8191, 8192])
def test_row_lengths(D, types):
    run(1, 11, D, types, gate="channel", act="tanh", seed=D)
    run(3, 9, D, types, gate="token", act="sigmoid", seed=D)


@pytest.mark.parametrize("T", [0, 1, 2, 7, 8, 9, 31, 300])
def test_numbers_of_rows(T):
    for P, D, types in ((1, 100, "bf16"), (3, 1031, "mixed"), (2, 4096, "bf16"), (5, 40, "f32")):
        run(P, T, D, types, gate="channel", act="sigmoid", seed=T)


def test_more_rows_than_the_machine_holds():
    """Every block takes several rows: the ring of rows and the running sums go round."""
    run(1, 300, 4100, "bf16", gate="channel", seed=3)
    run(2, 1201, 264, "mixed", gate="token", act="sigmoid", seed=4)
    run(1, 5003, 41, "f32", seed=5)


@pytest.mark.parametrize("kind,offset", [("rows", 0), ("rows", 8), ("rows", 1), ("padded", 0), ("aligned", 0), ("interleaved", 0),
                                         ("interleaved", 3)])
@pytest.mark.parametrize("D", [96, 101])
def test_strides_and_alignments(kind, offset, D):
    for types, P in itertools.product(TYPES, (1, 4)):
        run(P, 21, D, types, gate="token", act="tanh", kind=kind, offset=offset, seed=D)


def test_in_place_and_accumulated():
    for types in TYPES:
        for D in (512, 333):
            run(2, 37, D, types, gate="channel", in_place=True, accumulate=True, seed=9)
            run(1, 37, D, types, y=False, in_place=True, accumulate=True, seed=10)


def test_zero_rows_large_and_small_values():
    run(2, 9, 200, "f32", zero_row=True, seed=1)              # 1 / sqrt(0 + eps): nothing is divided by zero
    run(1, 9, 200, "f32", scale=1e15, eps=1e-5, seed=2, pre=True)
    run(1, 9, 200, "f32", scale=1e-15, eps=1e-12, seed=3)


def test_one_gain_for_all_workers():
    """Gains and a gate expanded over the workers, and their gradients summed over them; one row for all rows."""
    from paper_1905_10395_b200 import lm
    P, T, D = 3, 50, 160
    gen = torch.Generator().manual_seed(5)
    mk = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64).float()  # noqa: E731
    x, y, d_out, d_h = (mk(P, T, D) for _ in range(4))
    w_post, w_pre, gate = (mk(D) for _ in range(3))
    shared = lambda v: v.cuda()[None].expand(P, D)  # noqa: E731
    out, h, dx, dy = (torch.empty(P, T, D, device="cuda") for _ in range(4))
    dw = {k: torch.zeros(D, device="cuda") for k in ("dw_post", "dw_pre", "d_gate")}
    op = lm.BlockNorm(x=x.cuda(), y=y.cuda(), gate=shared(gate), w_post=shared(w_post), w_pre=shared(w_pre), out=out, h=h,
                      d_out=d_out.cuda(), d_h=d_h.cuda(), dx=dx, dy=dy, gate_act="sigmoid",
                      **{k: v[None].expand(P, D) for k, v in dw.items()})
    op.forward()
    op.backward()
    torch.cuda.synchronize()
    d = {k: v.double()[None].expand(P, D) for k, v in (("gate", gate), ("w_post", w_post), ("w_pre", w_pre))}
    want, _ = ref.blocknorm_backward(d_out.double(), d_h.double(), out.cpu().double(), y.double(), act="sigmoid", **d)
    for k, v in dw.items():
        w = want[k].sum(0)
        assert (v.cpu().double() - w).abs().max() <= 2.0 ** -14 * want[k].abs().sum(0).max() + 1e-4
    # one row of y for every token and worker
    row = mk(D)
    op = lm.BlockNorm(x=x.cuda(), y=row.cuda().expand(P, T, D), w_pre=shared(w_pre), out=out, h=h, post_norm=False)
    op.forward()
    torch.cuda.synchronize()
    assert (out.cpu().double() - (x.double() + row.double())).abs().max() < 1e-5


def test_not_finite_rows_stay_rows():
    """A row with an infinity or NaN is not finite afterwards; its neighbours are what they were."""
    from paper_1905_10395_b200 import lm
    T, D = 24, 333
    gen = torch.Generator().manual_seed(6)
    x, y = (torch.randn(1, T, D, generator=gen).to(torch.bfloat16) for _ in range(2))
    w = torch.ones(1, D).cuda()
    res = []
    for poison in (False, True):
        yy = y.clone()
        if poison:
            yy[0, 3, 0], yy[0, 7, D - 1], yy[0, 11, 100] = float("inf"), float("nan"), float("-inf")
        out, h = (torch.empty(1, T, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lm.BlockNorm(x=x.cuda(), y=yy.cuda(), w_post=w, w_pre=w, out=out, h=h).forward()
        torch.cuda.synchronize()
        res.append((out.cpu(), h.cpu()))
    bad = [3, 7, 11]
    good = [t for t in range(T) if t not in bad]
    for a, b in zip(*res):
        assert torch.equal(a[0, good], b[0, good])
        assert (~torch.isfinite(b[0, bad].float())).any(-1).all()


def test_same_inputs_same_bits():
    from paper_1905_10395_b200 import lm
    T, D = 2000, 1000
    gen = torch.Generator(device="cuda").manual_seed(7)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    out, y, d_out, d_h, w, g = mk(1, T, D), mk(1, T, D), mk(1, T, D), mk(1, T, D), mk(1, D), mk(1, D)
    r = [torch.rsqrt(v.square().mean(-1) + 1e-6) for v in (out, y)]
    got = []
    for _ in range(2):
        res = {k: torch.empty(1, T, D, device="cuda") for k in ("dx", "dy")}
        res.update({k: torch.empty(1, D, device="cuda") for k in ("d_gate", "dw_post", "dw_pre")})
        lm.BlockNorm(out=out, y=y, gate=g, w_post=w, w_pre=w, d_out=d_out, d_h=d_h, rstd_pre=r[0], rstd_post=r[1], **res).backward()
        torch.cuda.synchronize()
        got.append(res)
    assert all(torch.equal(got[0][k], got[1][k]) for k in got[0])


@pytest.mark.parametrize("D", [72, 75])
def test_gradient_against_differences(D):
    """The loss sum(c1 x') + sum(c2 h) along random directions: its central difference in 64 bits, error O(step^2), against the
    kernel's fp32 gradients."""
    from paper_1905_10395_b200 import lm
    P, T = 2, 6
    gen = torch.Generator().manual_seed(8)
    mk = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64).float().double()  # noqa: E731
    v = {"x": mk(P, T, D), "y": mk(P, T, D), "gate": mk(P, D), "w_post": mk(P, D), "w_pre": mk(P, D)}
    c1, c2 = mk(P, T, D), mk(P, T, D)
    opt = dict(act="tanh", alpha=0.8, beta=1.1, eps=1e-3)

    def loss(w):
        o, h = ref.blocknorm_forward(w["x"], w["y"], w["gate"], w["w_post"], w["w_pre"], **opt)
        return float((c1 * o).sum() + (c2 * h).sum())

    dev = {k: t.float().cuda() for k, t in v.items()}
    out, h, dx, dy = (torch.empty(P, T, D, device="cuda") for _ in range(4))
    dw = {k: torch.empty(P, D, device="cuda") for k in ("d_gate", "dw_post", "dw_pre")}
    op = lm.BlockNorm(out=out, h=h, d_out=c1.float().cuda(), d_h=c2.float().cuda(), dx=dx, dy=dy, gate_act="tanh", alpha=0.8,
                      beta=1.1, eps=1e-3, **dev, **dw)
    op.forward()
    op.backward()
    torch.cuda.synchronize()
    grads = {"x": dx, "y": dy, "gate": dw["d_gate"], "w_post": dw["dw_post"], "w_pre": dw["dw_pre"]}
    for k, g in grads.items():
        u = mk(*v[k].shape)
        e = 1e-5
        up, down = dict(v), dict(v)
        up[k], down[k] = v[k] + e * u, v[k] - e * u
        num = (loss(up) - loss(down)) / (2 * e)
        mine = float((g.cpu().double() * u).sum())
        size = float((g.cpu().double() * u).abs().sum())
        assert abs(num - mine) <= 1e-5 * size + 1e-6, (k, num, mine)
