"""Every form that the convolution, the scan and the orthogonalisation take by size, against 64 bits: the form is asked for, so that a
change of the rules that choose it does not leave one untested."""
import ctypes as C

import pytest
import torch

from tests import _lm_mixer_reference as ref
from tests._lm_reference import Guarded

pytestmark = pytest.mark.gpu


def _plan(op, name, n, *args):
    from paper_1905_10395_b200 import api
    out = (C.c_int32 * n)()
    assert getattr(api.lib(), f"lsgd_{name}_plan")(C.byref(op.desc), *args, out) == 0
    return list(out)


def _expect(plan, want):
    """The forms are those of 148 SMs."""
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        assert plan == want


# ------------------------------------------------------------------------------------------------ orthogonalisation
# columns of the three products' tiles (256: pairs of blocks), most tiles of a block or pair, blocks that share a contraction.  Sizes that no tile
# divides, results that are stored 8 values at a time, value by value, and transposed.
ORTHO = [((24, 500, 704), [256, 256, 256, 1, 1, 2, 1]), ((24, 500, 701), [256, 256, 256, 1, 1, 2, 1]), ((24, 701, 500), [256, 256, 256, 1, 1, 2, 1]),
         ((9, 1001, 1104), [256, 256, 256, 2, 2, 3, 1]), ((9, 1003, 1001), [256, 256, 256, 2, 2, 2, 1]), ((1, 2049, 4100), [256, 256, 128, 1, 1, 4, 1]),
         ((40, 300, 400), [128, 128, 128, 2, 2, 4, 1]), ((60, 263, 300), [128, 128, 128, 3, 3, 4, 1]), ((40, 401, 300), [128, 128, 128, 2, 2, 4, 1]),
         ((19, 260, 300), [128, 128, 64, 1, 1, 2, 1]), ((20, 200, 3000), [128, 64, 256, 1, 1, 4, 2]), ((2, 600, 20000), [128, 64, 256, 1, 1, 7, 4]),
         ((300, 100, 300), [128, 128, 128, 3, 3, 7, 1]), ((3, 1001, 333), [64, 64, 64, 1, 1, 1, 4]), ((8, 128, 128), [0] * 7)]


@pytest.mark.parametrize("shape,plan", ORTHO, ids=[str(s) for s, _ in ORTHO])
def test_orthogonalisation(shape, plan):
    """Bounds of test_gpu_lm_ortho_ranks.py for all singular values, and of test_gpu_lm_ortho.py for every value."""
    from paper_1905_10395_b200 import api, lm
    P, m, n = shape
    g = torch.randn(shape, generator=torch.Generator().manual_seed(n))
    wide = n % 8 == 0
    ld = n + (8 if wide else 3)
    out = Guarded(shape, (m * ld + (8 if wide else 5), ld, 1), torch.bfloat16, 0 if wide else 1)
    dev = g.cuda()
    op = lm.Orthogonalize(dev, out.view)
    _expect(_plan(op, "ortho", 7), plan)
    op.forward()
    first = out.view.clone()
    op.forward()
    torch.cuda.synchronize()
    assert api.lsgd_ortho_check_device() == 0
    assert torch.equal(first, out.view) and out.intact()
    want, _ = ref.ortho(dev.double())
    off, rms = first.double() - want, want.square().mean((1, 2), keepdim=True).sqrt()
    norm = torch.linalg.matrix_norm
    assert (norm(off) <= 2.0 ** -8 * norm(want)).all(), (norm(off) / norm(want)).max()
    assert (off.abs() <= 2.0 ** -4 * rms + 2.0 ** -8 * want.abs()).all()


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
@pytest.mark.parametrize("shape", [(2, 100, 200), (3, 120, 700), (24, 500, 701), (40, 401, 300)], ids=str)
def test_orthogonalisation_by_steps(shape, steps):
    """What X is rounded by is taken from the step before and left for the next one, but by the last: 1 to 6 of them."""
    from paper_1905_10395_b200 import lm
    dev = torch.randn(shape, generator=torch.Generator().manual_seed(steps)).cuda()
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    lm.Orthogonalize(dev, out, steps=steps).forward()
    want, _ = ref.ortho(dev.double(), steps=steps)
    norm = torch.linalg.matrix_norm
    assert (norm(out.double() - want) <= 2.0 ** -8 * norm(want)).all(), (norm(out.double() - want) / norm(want)).max()


# ------------------------------------------------------------------------------------------------ convolution
def _starts(P, T, S, gen):
    cut = torch.randint(2, T - 3, (P, S + 1), generator=gen).sort(1)[0].int()
    cut[:, 1] = cut[:, 0]                        # an empty one
    return cut


# (values a thread, rows a thread, warps of a last sum) forwards and backwards
CONV = [((8, 1181, 2052), "bf16", [4, 64, 0], [4, 64, 1]), ((8, 1021, 2050), "bf16", [2, 24, 0], [2, 64, 1]), ((8, 1021, 2051), "bf16", [1, 24, 0], [1, 64, 1]),
        ((8, 1021, 2052), "f32", [2, 24, 0], [2, 64, 1]), ((8, 1021, 2051), "f32", [1, 24, 0], [1, 64, 1]), ((1, 5000, 64), "bf16", [2, 8, 0], [2, 8, 8]),
        ((1, 20001, 100), "bf16", [2, 16, 0], [2, 16, 8]), ((2, 30001, 24), "f32", [2, 16, 0], [2, 32, 8])]


@pytest.mark.parametrize("shape,dtype,fwd,bwd", CONV, ids=[f"{s}-{t}" for s, t, _, _ in CONV])
@pytest.mark.parametrize("W", [4, 3])
@pytest.mark.parametrize("where", ["equal", "ragged", "ragged with states"])
def test_convolution(shape, dtype, fwd, bwd, W, where):
    """Bounds of test_gpu_lm_conv.py; sums over T rows add T 2^-24 of the terms at most."""
    from paper_1905_10395_b200 import lm
    P, T, D = shape
    A = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator().manual_seed(T + W)
    dev = torch.Generator(device="cuda").manual_seed(T + W)
    r = lambda *s, d=torch.float32: torch.randn(s, generator=dev, device="cuda").to(d)  # noqa: E731
    starts = None if where == "equal" else _starts(P, T, 9, gen)
    S = 1 if starts is None else 9
    edges = ref.edges_of(P, T, S, starts)
    live = torch.zeros((P, T), dtype=torch.bool)
    for p in range(P):
        live[p, edges[p][0]:edges[p][-1]] = True
    live = live.cuda()
    x, up, w, bias = r(P, T, D, d=A), r(P, T, D, d=A), r(P, D, W), r(P, D)
    x[~live], up[~live] = float("nan"), float("nan")
    kept = r(P, S, W - 1, D, d=A) if where == "ragged with states" else None
    old = None if kept is None else kept.clone()
    out = torch.full_like(x, 7.0)
    grads = {} if kept is not None else {"d_out": up, "dx": torch.full_like(x, 7.0), "dw": torch.empty_like(w), "d_bias": torch.empty_like(bias)}
    op = lm.CausalConv(x, w, bias=bias, out=out, state=kept, starts=None if starts is None else starts.cuda(), **grads)
    _expect(_plan(op, "conv", 3, 0), fwd)
    op.forward()
    if grads:
        _expect(_plan(op, "conv", 3, 1), bwd)
        op.backward()
    with torch.device("cuda"):
        got, size = ref.conv(x.double(), w.double(), bias.double(), None if old is None else old.double(), up.double() if grads else None, edges)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    for k, v in {"out": out, **{k: v for k, v in grads.items() if k != "d_out"}}.items():
        want, mag, rel = got.pop(k), size.pop(k), 2.0 ** -17
        if k in ("out", "dx"):
            assert (v[~live] == 7.0).all(), k
            v, want, mag = v[live], want[live], mag[live]
            bound = rel * mag + half * want.abs()
        else:
            bound = (rel + T * 2.0 ** -24) * mag
        bad = ~((v.double() - want).abs() <= bound + 1e-35)
        assert not bad.any(), (k, int(bad.sum()))
    if kept is not None:
        assert torch.equal(kept, got["state"].to(A))


# ------------------------------------------------------------------------------------------------ scan
@pytest.fixture
def scans(monkeypatch):
    """The operators that a test makes."""
    from paper_1905_10395_b200 import lm
    made, real = [], lm.SelectiveScan

    def make(*a, **k):
        made.append(real(*a, **k))
        return made[-1]

    monkeypatch.setattr(lm, "SelectiveScan", make)
    return made


# lanes a channel, chains of a worker, rows of a chain that are split, single tokens
SCAN = [(dict(P=160, T=12, D=20, N=33), [16, 1, 0, 0]), (dict(P=160, T=12, D=24, N=64), [16, 1, 0, 0]), (dict(P=150, T=40, D=16, N=32, dtype="f32"), [8, 1, 0, 0]),
        (dict(P=40, T=48, D=20, N=64, S=4), [16, 4, 0, 0]), (dict(P=3, T=600, D=20, N=24, S=100), [8, 50, 0, 0]), (dict(P=3, T=400, D=40, N=5, S=100), [2, 100, 0, 0]),
        (dict(P=1, T=1000, D=9, N=40, dtype="f32"), [16, 16, 64, 0]), (dict(P=1, T=1000, D=33, N=24), [8, 16, 64, 0]), (dict(P=2, T=700, D=70, N=8), [2, 11, 64, 0]),
        (dict(P=1, T=200, D=700, N=16), [4, 4, 64, 0]), (dict(P=1, T=200, D=704, N=16, dtype="f32"), [4, 4, 64, 0])]


@pytest.mark.parametrize("case,plan", SCAN, ids=[str(c) for c, _ in SCAN])
def test_scan(scans, case, plan):
    from tests.test_gpu_lm_scan import run
    run(**case, seed=case["T"])
    _expect(_plan(scans[-1], "scan", 4, 1), plan)


@pytest.mark.parametrize("N", [24, 40])
def test_scan_of_ragged_sequences_with_many_states(scans, N):
    """Rows split into chains, with sequences that begin in front of, at and behind their ends; chains of whole sequences."""
    from tests.test_gpu_lm_scan import run
    run(1, 500, 9, N, "f32", starts=torch.tensor([3, 64, 64, 65, 300, 301, 384, 490], dtype=torch.int32))
    assert _plan(scans[-1], "scan", 4, 1)[2] > 0
    cut = torch.randint(0, 33, (150, 4), generator=torch.Generator().manual_seed(N)).sort(1)[0].int()
    run(150, 32, 12, N, starts=cut)
    assert _plan(scans[-1], "scan", 4, 1)[2] == 0


@pytest.mark.parametrize("N", [3, 16, 40])
def test_scan_of_single_tokens(scans, N):
    from tests.test_gpu_lm_scan import run
    run(1, 70, 500, N, S=70, state=True, grads=False)
    _expect(_plan(scans[-1], "scan", 4, 0)[3:], [1])
