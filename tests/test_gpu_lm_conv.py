"""GPU check of the causal convolution (lsgd_conv_*) against its 64-bit restatement: types, widths, sequences, states, strides,
shared operands, and the gradient against differences.

Bounds.  pre is a chain of W + 1 <= 5 roundings, the activation (fast exponential, quotient) is within 2^-19: 2^-17 of the
magnitudes with room for the gradient's further products; sums over T <= 700 rows add at most 700 2^-24 < 2^-14 of the terms.  Half a
step (2^-8 of the value) where a result is stored in bf16."""
import pytest
import torch

from tests import _lm_mixer_reference as ref
from tests._lm_reference import Guarded

pytestmark = pytest.mark.gpu

REL, SUM = 2.0 ** -17, 2.0 ** -14
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(name, got, want, size, rel):
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    got = got.double().cpu()
    bound = rel * size + half * want.abs() + 1e-35
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {((got - want).abs() / bound)[bad].max():.3g} of the bound"


def strides(kind, P, T, D):
    return {"rows": (T * D, D, 1), "padded": (T * (D + 5) + 3, D + 5, 1), "aligned": (T * ((D + 15) // 8 * 8), (D + 15) // 8 * 8, 1),
            "interleaved": (D, P * D, 1)}[kind]


def draw(gen, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(dtype)


def vectors(shape, inner, fill, shared, offset=0):
    """A guarded fp32 buffer of [P, ...] whose rows are `inner` apart; shared: one worker's, expanded over them."""
    n = 1 if shared else shape[0]
    g = Guarded((n, *shape[1:]), inner, torch.float32, offset, fill[:n])
    if shared:
        g.view = g.view.expand(shape)
    return g


def live_rows(edges, P, T):
    live = torch.zeros((P, T), dtype=torch.bool)
    for p in range(P):
        live[p, edges[p][0]:max(edges[p][-1], edges[p][0])] = True
    return live


def run(P, T, D, W=4, dtype="bf16", S=None, starts=None, state=False, act="silu", bias=True, kind="rows", offset=0, grads=True,
        accumulate=False, shared=False, seed=0):
    from paper_1905_10395_b200 import lm
    A = TYPES[dtype]
    gen = torch.Generator().manual_seed(seed)
    n_seq = S or (starts.shape[-1] - 1 if starts is not None else 1)
    edges = ref.edges_of(P, T, n_seq, starts)
    live = live_rows(edges, P, T)
    host = {"x": draw(gen, (P, T, D), A), "w": draw(gen, (1 if shared else P, D, W)).expand(P, D, W)}
    if bias:
        host["bias"] = draw(gen, (1 if shared else P, D)).expand(P, D)
    if state:
        host["state"] = draw(gen, (P, n_seq, W - 1, D), A)
    if grads:
        host["d_out"] = draw(gen, (P, T, D), A)
    for k in ("x", "d_out"):            # what no sequence holds is not read
        if k in host:
            host[k][~live] = float("nan")
    st = strides(kind, P, T, D)
    dev = {k: Guarded((P, T, D), st, A, offset, host[k]) for k in ("x", "d_out") if k in host}
    dev["w"] = vectors((P, D, W), (D * (W + 1) + 2, W + 1, 1), host["w"], shared, 1)
    if bias:
        dev["bias"] = vectors((P, D), (D + 3, 1), host["bias"], shared, 1)
    rows = {"out": Guarded((P, T, D), st, A, offset)}
    kept = host["state"].cuda() if state else None
    kw, start = {}, {}
    if grads:
        rows["dx"] = Guarded((P, T, D), st, A, offset)
        start["dw"] = draw(gen, (1 if shared else P, D, W)).expand(P, D, W)
        rows["dw"] = vectors((P, D, W), (D * (W + 2), W + 2, 1), start["dw"], shared)
        if bias:
            start["d_bias"] = draw(gen, (1 if shared else P, D)).expand(P, D)
            rows["d_bias"] = vectors((P, D), (D + 1, 1), start["d_bias"], shared)
        kw = {k: rows[k].view for k in rows if k != "out"} | {"d_out": dev["d_out"].view}
    op = lm.CausalConv(dev["x"].view, dev["w"].view, bias=dev["bias"].view if bias else None, out=rows["out"].view, state=kept, act=act,
                       sequences=S, starts=starts.cuda() if starts is not None else None, accumulate=accumulate, **kw)
    before = {k: rows[k].view.cpu().clone() for k in rows}
    op.forward()
    if grads:
        op.backward()
    torch.cuda.synchronize()
    f64 = {k: v.double() for k, v in host.items()}
    got, size = ref.conv(f64["x"], f64["w"], f64.get("bias"), f64.get("state"), f64.get("d_out"), edges, act)
    for k in ("out", "dx"):
        if k in rows:
            mine = rows[k].view.cpu()
            close(k, mine[live], got[k][live], size[k][live], REL)
            assert torch.equal(mine[~live].view(torch.uint8), before[k][~live].view(torch.uint8)), f"{k}: rows of no sequence were written"
    if state:
        assert torch.equal(kept.cpu(), got["state"].to(A))
    for k in ("dw", "d_bias"):
        if k in rows:
            want, mag = got[k], size[k]
            if shared:
                want, mag = want.sum(0, keepdim=True).expand_as(want), mag.sum(0, keepdim=True).expand_as(mag)
            if accumulate:
                want, mag = want + start[k].double(), mag + start[k].double().abs()
            close(k, rows[k].view, want, mag, SUM)
    for g in (*dev.values(), *rows.values()):
        assert g.intact()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [1, 2, 3, 4])
@pytest.mark.parametrize("D,kind,offset", [(8, "rows", 0), (132, "aligned", 0), (250, "padded", 1), (17, "interleaved", 0)])
def test_widths_and_rows(dtype, W, D, kind, offset):
    run(2, 100, D, W, dtype, kind=kind, offset=offset, bias=W != 2, act="identity" if W == 3 else "silu", accumulate=W == 4, seed=W)


@pytest.mark.parametrize("T", [0, 1, 2, 3, 4, 5, 7, 8, 9, 31, 32, 33, 63, 65, 127, 257, 700])
def test_lengths(T):
    run(1, T, 36, seed=T)
    run(3, T, 20, 3, "f32", seed=T + 1)
    run(1, T, 8, state=True, grads=False, seed=T + 2)


RAGGED = [[0, 0, 1, 3, 3, 6, 50, 51, 52, 90], [5, 20, 20, 20, 60], [0, 90], [90, 90], [0, 0, 0], [40, 41], [89, 90, 90]]


@pytest.mark.parametrize("starts", RAGGED, ids=str)
@pytest.mark.parametrize("state", [False, True])
def test_ragged_sequences(starts, state):
    run(2, 90, 44, starts=torch.tensor(starts, dtype=torch.int32), state=state, grads=not state, seed=len(starts))


def test_starts_of_every_worker():
    starts = torch.tensor([[0, 10, 10, 64], [3, 4, 30, 31], [64, 64, 64, 64]], dtype=torch.int32)
    run(3, 64, 40, starts=starts, dtype="f32")
    run(3, 64, 40, 3, starts=starts, state=True, grads=False)


@pytest.mark.parametrize("S", [1, 2, 5, 20, 60])
def test_equal_sequences_and_states(S):
    run(2, 60, 68, S=S, state=True, grads=False, seed=S)
    run(2, 60, 7, 2, "f32", S=S, state=True, grads=False, kind="padded", seed=S + 1)
    run(2, 60, 68, S=S, seed=S + 2)


def test_shared_operands():
    run(4, 50, 24, shared=True)
    run(4, 50, 24, shared=True, accumulate=True, dtype="f32", kind="padded")


def test_prompt_then_tokens():
    """A sequence taken whole gives what a prompt and then single tokens give, bit for bit."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(3)
    x, w = draw(gen, (1, 40, 64), torch.bfloat16).cuda(), draw(gen, (1, 64, 4)).cuda()
    whole = torch.empty_like(x)
    lm.CausalConv(x, w, out=whole).forward()
    state, parts = torch.zeros((1, 1, 3, 64), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    lm.CausalConv(x[:, :33], w, out=parts[:, :33], state=state).forward()
    for t in range(33, 40):
        lm.CausalConv(x[:, t:t + 1], w, out=parts[:, t:t + 1], state=state).forward()
    torch.cuda.synchronize()
    assert torch.equal(whole, parts) and torch.equal(state[0, 0], x[0, 37:])


def test_infinite_inputs_stay_where_they_are_read():
    """A width of 2: an infinite input three rows back is not multiplied by a weight of zero."""
    from paper_1905_10395_b200 import lm
    x, w = torch.ones((1, 32, 4), device="cuda"), torch.ones((1, 4, 2), device="cuda")
    x[0, 10] = float("inf")
    out = torch.empty_like(x)
    lm.CausalConv(x, w, out=out, act="identity").forward()
    torch.cuda.synchronize()
    assert torch.isinf(out[0, 10:12]).all() and torch.equal(out[0, 12:], torch.full_like(out[0, 12:], 2.0))


def test_gradient_against_differences():
    """Central differences of the kernel's own forward pass in fp32, step 2^-6: the third derivative leaves below 2^-12 of the values'
    scale (|act'''| < 1), rounding 2^-24 / 2^-6 = 2^-18 of the outputs' sum: 2^-8 of the gradient's norm is above both."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(9)
    P, T, D, W = 1, 24, 8, 4
    x, w, bias = draw(gen, (P, T, D)).cuda(), draw(gen, (P, D, W)).cuda(), draw(gen, (P, D)).cuda()
    up = draw(gen, (P, T, D)).cuda()
    out, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(bias)
    op = lm.CausalConv(x, w, bias=bias, out=out, d_out=up, dx=dx, dw=dw, d_bias=db, sequences=2)
    op.backward()
    for t, g in ((x, dx), (w, dw), (bias, db)):
        want = torch.zeros_like(g)
        for i in range(t.numel()):
            old, at = float(t.view(-1)[i]), []
            for h in (2.0 ** -6, -2.0 ** -6):
                t.view(-1)[i] = old + h
                op.forward()
                at.append(float((out.double() * up.double()).sum()))
            t.view(-1)[i] = old
            want.view(-1)[i] = (at[0] - at[1]) / 2 ** -5
        assert (want - g).norm() <= 2.0 ** -8 * g.norm()
