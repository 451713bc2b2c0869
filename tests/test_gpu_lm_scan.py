"""GPU check of the selective state space scan (lsgd_scan_*) against its 64-bit restatement: types, numbers of states, sequences,
states, strides, shared operands, chains that split the rows, and the gradient against differences.

Bounds.  Every row's decay exp(delta A) is within 2^-22 by the exponential and within delta |A| 2^-21 by its argument; over the rows
between two tokens the first add up to T 2^-22 and the second to e^-s s 2^-21 < 2^-22.  The other factors and sums are chains of
fewer than 64 + D roundings of 2^-24, the activations are within 2^-18 of their magnitudes: (T + D + 64) 2^-22 of the magnitudes holds
all of them, twice that for gradients, in which two such chains meet.  Half a step (2^-8 of the value) where a result is stored
in bf16."""
import pytest
import torch

from tests import _lm_mixer_reference as ref
from tests._lm_reference import Guarded
from tests.test_gpu_lm_conv import RAGGED, TYPES, close, draw, live_rows, strides, vectors

pytestmark = pytest.mark.gpu

ROWS = {"x": "D", "dt": "D", "z": "D", "d_out": "D", "b": "N", "c": "N"}
GRADS = {"d_x": "D", "d_dt": "D", "d_z": "D", "d_b": "N", "d_c": "N"}


def run(P, T, D, N=16, dtype="bf16", S=None, starts=None, state=False, gate=True, skip=True, bias=True, kind="rows", offset=0,
        grads=True, accumulate=False, shared=False, seed=0):
    from paper_1905_10395_b200 import lm
    A = TYPES[dtype]
    gen = torch.Generator().manual_seed(seed)
    n_seq = S or (starts.shape[-1] - 1 if starts is not None else 1)
    edges = ref.edges_of(P, T, n_seq, starts)
    live = live_rows(edges, P, T)
    size_of = {"D": D, "N": N}
    one = 1 if shared else P
    host = {k: draw(gen, (P, T, size_of[n]), A) for k, n in ROWS.items() if (k != "z" or gate) and (k != "d_out" or grads)}
    host["a_log"] = draw(gen, (one, D, N), scale=0.7).expand(P, D, N)
    if skip:
        host["skip"] = draw(gen, (one, D)).expand(P, D)
    if bias:
        host["dt_bias"] = (draw(gen, (one, D)) - 2).expand(P, D)
    if state:
        host["state"] = draw(gen, (P, n_seq, D, N))
    for k in ROWS:
        if k in host:
            host[k][~live] = float("nan")
    where = lambda n: strides(kind, P, T, size_of[n])  # noqa: E731
    dev = {k: Guarded((P, T, size_of[n]), where(n), A, offset, host[k]) for k, n in ROWS.items() if k in host}
    dev["a_log"] = vectors((P, D, N), (D * (N + 1) + 2, N + 1, 1), host["a_log"], shared, 1)
    for k in ("skip", "dt_bias"):
        if k in host:
            dev[k] = vectors((P, D), (D + 3, 1), host[k], shared, 1)
    rows = {"out": Guarded((P, T, D), where("D"), A, offset)}
    start = {}
    if grads:
        for k, n in GRADS.items():
            if k != "d_z" or gate:
                rows[k] = Guarded((P, T, size_of[n]), where(n), A, offset)
        start["d_a_log"] = draw(gen, (one, D, N)).expand(P, D, N)
        rows["d_a_log"] = vectors((P, D, N), (D * (N + 2), N + 2, 1), start["d_a_log"], shared)
        for k in ("skip", "dt_bias"):
            if k in host:
                start["d_" + k] = draw(gen, (one, D)).expand(P, D)
                rows["d_" + k] = vectors((P, D), (D + 1, 1), start["d_" + k], shared)
    kept = host["state"].cuda() if state else None
    view = lambda k: dev[k].view if k in dev else None  # noqa: E731
    op = lm.SelectiveScan(view("x"), view("dt"), view("a_log"), view("b"), view("c"), z=view("z"), skip=view("skip"),
                          dt_bias=view("dt_bias"), state=kept, d_out=view("d_out"), sequences=S,
                          starts=starts.cuda() if starts is not None else None, accumulate=accumulate,
                          **{k: v.view for k, v in rows.items()})
    before = {k: rows[k].view.cpu().clone() for k in rows}
    op.forward()
    if grads:
        op.backward()
    torch.cuda.synchronize()
    f64 = {k: v.double() for k, v in host.items()}
    got, size = ref.scan(f64["x"], f64["dt"], f64["a_log"], f64["b"], f64["c"], f64.get("z"), f64.get("skip"), f64.get("dt_bias"),
                         f64.get("state"), f64.get("d_out"), edges)
    rel = (T + D + 64) * 2.0 ** -22
    for k in ("out", *GRADS):
        if k in rows:
            mine = rows[k].view.cpu()
            close(k, mine[live], got[k][live], size[k][live], rel if k == "out" else 2 * rel)
            assert torch.equal(mine[~live].view(torch.uint8), before[k][~live].view(torch.uint8)), f"{k}: rows of no sequence were written"
    if state:
        close("state", kept, got["state"], size["state"], rel)
        for p in range(P):
            for i in range(n_seq):
                if edges[p][i + 1] <= edges[p][i]:
                    assert torch.equal(kept[p, i].cpu(), host["state"][p, i])
    for k in start:
        want, mag = got[k], size[k]
        if shared:
            want, mag = want.sum(0, keepdim=True).expand_as(want), mag.sum(0, keepdim=True).expand_as(mag)
        if accumulate:
            want, mag = want + start[k].double(), mag + start[k].double().abs()
        close(k, rows[k].view, want, mag, 2 * rel)
    for g in (*dev.values(), *rows.values()):
        assert g.intact()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 3, 4, 8, 9, 13, 16, 17, 32, 33, 50, 64])
def test_numbers_of_states(dtype, N):
    run(2, 70, 72, N, dtype, seed=N)
    run(1, 40, 21, N, dtype, state=True, grads=False, S=2, seed=N + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,kind,offset", [(8, "rows", 0), (136, "aligned", 0), (250, "padded", 1), (17, "interleaved", 0), (65, "rows", 3)])
def test_rows(dtype, D, kind, offset):
    run(2, 50, D, 16, dtype, kind=kind, offset=offset, gate=D != 17, skip=D != 65, bias=D != 8, accumulate=D == 250, seed=D)


@pytest.mark.parametrize("T", [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129, 300])
def test_lengths(T):
    run(1, T, 24, seed=T)
    run(3, T, 16, 5, "f32", seed=T + 1)
    run(1, T, 40, state=True, grads=False, seed=T + 2)


@pytest.mark.parametrize("starts", RAGGED, ids=str)
@pytest.mark.parametrize("state", [False, True])
def test_ragged_sequences(starts, state):
    run(2, 90, 44, starts=torch.tensor(starts, dtype=torch.int32), state=state, grads=not state, seed=len(starts))


def test_starts_of_every_worker():
    starts = torch.tensor([[0, 10, 10, 64], [3, 4, 30, 31], [64, 64, 64, 64]], dtype=torch.int32)
    run(3, 64, 40, starts=starts, dtype="f32")
    run(3, 64, 40, starts=starts, state=True, grads=False)


@pytest.mark.parametrize("S", [1, 2, 5, 20, 60])
def test_equal_sequences_and_states(S):
    run(2, 60, 68, S=S, state=True, grads=False, seed=S)
    run(2, 60, 7, 11, "f32", S=S, state=True, grads=False, kind="padded", seed=S + 1)
    run(2, 60, 68, S=S, seed=S + 2)


def test_shared_operands():
    run(4, 50, 24, shared=True)
    run(4, 50, 24, 9, shared=True, accumulate=True, dtype="f32", kind="padded")


@pytest.mark.parametrize("P,S", [(160, 1), (40, 4), (3, 100), (200, 3)])
def test_chains_of_whole_sequences(P, S):
    """Enough workers or sequences to fill the SMs: chains are runs of sequences, some of several."""
    run(P, 12 * S, 20, S=S, seed=P)


@pytest.mark.parametrize("starts", [None, [0, 2000], [3, 64, 64, 65, 700, 701, 1408, 1990], [0] + [64 * i for i in range(1, 31)]], ids=str)
@pytest.mark.parametrize("state", [False, True])
def test_split_rows(starts, state):
    """Few channels and many rows: chains of equal runs of rows, with sequences that begin at, in front of and behind their ends."""
    run(1, 2000, 9, 16, "f32", starts=torch.tensor(starts, dtype=torch.int32) if starts else None, state=state, grads=not state)


def test_ragged_sequences_of_many_workers():
    cut = torch.randint(0, 65, (150, 6), generator=torch.Generator().manual_seed(5)).sort(1)[0].int()
    run(150, 64, 12, starts=cut)
    run(150, 64, 12, starts=cut, state=True, grads=False)


def test_prompt_then_tokens():
    """A sequence taken whole gives what a prompt and then single tokens give (bounds as above: the decays of 64 rows)."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(3)
    T, D, N = 64, 72, 16
    x, dt, z = (draw(gen, (1, T, D)).cuda() for _ in range(3))
    b, c = (draw(gen, (1, T, N)).cuda() for _ in range(2))
    a_log, skip = draw(gen, (1, D, N)).cuda(), draw(gen, (1, D)).cuda()
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    lm.SelectiveScan(x, dt, a_log, b, c, z=z, skip=skip, out=whole).forward()
    state = torch.zeros((1, 1, D, N), device="cuda")
    cut = lambda lo, hi: [v[:, lo:hi] for v in (x, dt, b, c, z, parts)]  # noqa: E731
    for lo, hi in [(0, 50)] + [(t, t + 1) for t in range(50, T)]:
        xx, dd, bb, cc, zz, oo = cut(lo, hi)
        lm.SelectiveScan(xx, dd, a_log, bb, cc, z=zz, skip=skip, out=oo, state=state).forward()
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu()  # noqa: E731
    _, size = ref.scan(f(x), f(dt), f(a_log), f(b), f(c), f(z), f(skip), None, None, None, [[0, T]])
    assert ((whole - parts).abs().double().cpu() <= 2 * (T + D + 64) * 2.0 ** -22 * size["out"]).all()


def test_a_sequence_that_overflows_leaves_its_neighbours():
    """Infinite values of one sequence do not reach the next one's rows, states or gradients."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(4)
    T, D, N = 48, 16, 16
    x, dt, d_out = (draw(gen, (1, T, D)).cuda() for _ in range(3))
    b, c, a_log = draw(gen, (1, T, N)).cuda(), draw(gen, (1, T, N)).cuda(), draw(gen, (1, D, N)).cuda()

    def go():
        out = {k: torch.zeros_like(v) for k, v in (("out", x), ("d_x", x), ("d_dt", x), ("d_b", b), ("d_c", c), ("d_a_log", a_log))}
        op = lm.SelectiveScan(x, dt, a_log, b, c, d_out=d_out, sequences=3, **out)
        op.forward()
        op.backward()
        torch.cuda.synchronize()
        return out

    clean = go()
    x[0, 20], d_out[0, 25] = float("inf"), float("inf")
    dirty = go()
    for k in ("out", "d_x", "d_dt", "d_b", "d_c"):
        assert torch.equal(clean[k][0, :16], dirty[k][0, :16]) and torch.equal(clean[k][0, 32:], dirty[k][0, 32:]), k
    assert not torch.isfinite(dirty["out"][0, 20:32]).all()


@pytest.mark.parametrize("split", [False, True])
def test_gradient_against_differences(split):
    """Central differences of the kernel's own forward pass in fp32, step 2^-6, of 40 entries of every input (of 600 rows where they
    are split: the first and last rows' too): rounding leaves (T + 64) 2^-22 / 2^-6 of the outputs' sum, the third derivative 2^-12 of
    the values' scale; 2 % of the differences' norm is above both."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(9)
    P, T, D, N = 1, 600 if split else 20, 8, 5
    x, dt, z, up = (draw(gen, (P, T, D)).cuda() for _ in range(4))
    b, c = draw(gen, (P, T, N)).cuda(), draw(gen, (P, T, N)).cuda()
    a_log, skip, bias = draw(gen, (P, D, N), scale=0.5).cuda(), draw(gen, (P, D)).cuda(), draw(gen, (P, D)).cuda()
    ins = {"x": x, "dt": dt, "z": z, "b": b, "c": c, "a_log": a_log, "skip": skip, "dt_bias": bias}
    grads = {"d_" + k: torch.empty_like(v) for k, v in ins.items()}
    out = torch.empty_like(x)
    op = lm.SelectiveScan(x, dt, a_log, b, c, z=z, skip=skip, dt_bias=bias, out=out, d_out=up, sequences=2, **grads)
    op.forward()
    op.backward()
    for k, t in ins.items():
        g = grads["d_" + k].view(-1)
        pick = torch.randperm(t.numel(), generator=gen)[:40].tolist() + [0, t.numel() - 1]
        want = []
        for i in pick:
            old, at = float(t.view(-1)[i]), []
            for h in (2.0 ** -6, -2.0 ** -6):
                t.view(-1)[i] = old + h
                op.forward()
                at.append(float((out.double() * up.double()).sum()))
            t.view(-1)[i] = old
            want.append((at[0] - at[1]) / 2 ** -5)
        want, mine = torch.tensor(want), g[pick].cpu()
        assert (want - mine).norm() <= 0.02 * want.norm(), k
