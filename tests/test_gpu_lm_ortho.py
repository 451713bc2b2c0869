"""GPU check of the orthogonalised updates (lsgd_ortho) against their 64-bit restatement: sizes, orientations, types, strides,
momentum, captured calls.

Bounds.  A step stores G, Q and X with an error of at most 2^-11 of each value, independent from entry to entry, so about 2^-12 in
the norm; through b G + c G G (|b| + 2 |c| < 9, against values that the step lets grow by up to 3.4) that is below 2^-9 of X's norm a
step for matrices whose singular values are within a factor of some tens of each other, and five steps add up in the squares
to below 2^-7.8; bf16's rounding is 2^-9.  A matrix is held to 2^-6.5 in the norm and every value to 2^-4 of the root mean square (the
largest of a million such errors is below 6 of their standard deviations of 2^-7.8)."""
import pytest
import torch

from tests import _lm_mixer_reference as ref
from tests._lm_reference import Guarded

pytestmark = pytest.mark.gpu

NORM, EACH = 2.0 ** -6.5, 2.0 ** -4


def close(got, want):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    for p in range(got.shape[0]):
        rms = want[p].square().mean().sqrt()
        off = got[p] - want[p]
        assert off.norm() <= NORM * want[p].norm() + 1e-30, (p, (off.norm() / want[p].norm()).item())
        assert (off.abs() <= EACH * rms + 2.0 ** -8 * want[p].abs()).all(), (p, (off.abs().max() / rms).item())


def run(P, m, n, dtype=torch.float32, momentum=False, nesterov=True, kind="rows", offset=0, steps=5, scale=1.0, size=1e-3, seed=0, **kw):
    from paper_1905_10395_b200 import api, lm
    gen = torch.Generator().manual_seed(seed)
    strides = {"rows": (m * n, n, 1), "padded": (m * (n + 5) + 3, n + 5, 1), "interleaved": (n, P * n, 1)}[kind]
    g = (torch.randn((P, m, n), generator=gen, dtype=torch.float64) * size).to(dtype)
    grad = Guarded((P, m, n), strides, dtype, offset, g)
    out = Guarded((P, m, n), strides, torch.bfloat16, offset)
    M = (torch.randn((P, m, n), generator=gen, dtype=torch.float64) * 3 * size).float() if momentum else None
    mom = Guarded((P, m, n), strides, torch.float32, offset, M) if momentum else None
    op = lm.Orthogonalize(grad.view, out.view, momentum=mom.view if momentum else None, nesterov=nesterov, steps=steps, scale=scale, **kw)
    op.forward()
    torch.cuda.synchronize()
    flag = api.C.c_uint32()
    assert api.lib().lsgd_ortho_check_device(api.C.byref(flag)) == 0
    want, new = ref.ortho(g.double(), M.double() if momentum else None, nesterov=nesterov, steps=steps, scale=scale, **kw)
    close(out.view, want)
    if momentum:
        assert ((mom.view.double().cpu() - new).abs() <= 2.0 ** -23 * (new.abs() + g.double().abs())).all()
    for b in (grad, out, mom):
        assert b is None or b.intact()
    return op, out


@pytest.mark.parametrize("m,n", [(1, 1), (1, 7), (7, 1), (2, 3), (16, 16), (33, 20), (63, 65), (64, 128), (128, 128), (128, 129), (130, 40),
                                 (200, 200), (256, 256), (257, 300), (100, 1000), (1000, 100), (384, 1024)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sizes(m, n, dtype):
    run(2, m, n, dtype, momentum=dtype == torch.float32, seed=m + n)


@pytest.mark.parametrize("kind,offset", [("rows", 0), ("rows", 3), ("padded", 1), ("interleaved", 0)])
@pytest.mark.parametrize("m,n", [(70, 150), (150, 70), (72, 64)])
def test_rows(kind, offset, m, n):
    run(3, m, n, kind=kind, offset=offset, momentum=True, nesterov=offset == 0, seed=offset)


@pytest.mark.parametrize("P,m,n", [(1, 1000, 700), (12, 256, 512), (40, 128, 96), (5, 600, 600), (1, 512, 2048)])
def test_many_tiles(P, m, n):
    run(P, m, n, seed=P)


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 7])
def test_steps(steps):
    run(2, 90, 140, steps=steps, scale=0.3, momentum=True)
    run(2, 300, 260, steps=steps, scale=-2.0)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e3, 1e15])
def test_magnitudes(size):
    """The norm is a sum in 64 bits: squares leave fp32's range, X does not."""
    run(2, 60, 90, size=size, eps=0.0)


def test_other_polynomials():
    """The classical third-order one, whose steps keep singular values below 1."""
    run(2, 80, 200, coefficients=(1.5, -0.5, 0.0), steps=8)
    run(2, 200, 300, coefficients=(1.875, -1.25, 0.375), steps=6)


def test_zero_and_not_finite_matrices():
    from paper_1905_10395_b200 import lm
    for eps in (1e-7, 0.0):
        for m, n in ((50, 90), (300, 200)):
            g = torch.randn(4, m, n, generator=torch.Generator().manual_seed(0)).cuda()
            g[1] = 0
            g[2, m // 2, 3] = float("nan")
            g[3, 0, 0] = float("inf")
            out = torch.empty((4, m, n), dtype=torch.bfloat16, device="cuda")
            lm.Orthogonalize(g, out, eps=eps).forward()
            torch.cuda.synchronize()
            assert torch.isfinite(out[0]).all() and (out[1] == 0).all()
            assert torch.isnan(out[2]).all() and torch.isnan(out[3]).all()


def test_rows_of_zeros_stay_zero():
    """A matrix padded with rows and columns of zeros gives what the matrix gives, and zeros."""
    g = torch.randn(1, 100, 60, generator=torch.Generator().manual_seed(2))
    g[0, 80:] = 0
    g[0, :, 50:] = 0
    from paper_1905_10395_b200 import lm
    out = torch.empty((1, 100, 60), dtype=torch.bfloat16, device="cuda")
    lm.Orthogonalize(g.cuda(), out).forward()
    torch.cuda.synchronize()
    assert (out[0, 80:] == 0).all() and (out[0, :, 50:] == 0).all()
    close(out[:, :80, :50], ref.ortho(g[:, :80, :50].double())[0])


def test_same_bits_and_capture():
    """Twice the same inputs give the same bits; a captured call replays on new contents, with its momentum moved each time."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(5)
    for m, n in ((64, 100), (500, 300)):
        g, M = torch.randn(3, m, n, generator=gen).cuda(), torch.randn(3, m, n, generator=gen).cuda()
        out = torch.empty((3, m, n), dtype=torch.bfloat16, device="cuda")
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            mom = M.clone()
            op = lm.Orthogonalize(g, out, momentum=mom)
            op.forward()
            first = out.clone()
            mom.copy_(M)
            graph = torch.cuda.CUDAGraph()
            s.synchronize()
            with torch.cuda.graph(graph, stream=s):
                op.forward()
            out.zero_()
            graph.replay()
            assert torch.equal(out, first)
            graph.replay()
        torch.cuda.synchronize()
        want = M.double().cpu()
        for _ in range(2):
            exact, want = ref.ortho(g.double().cpu(), want)
        close(out, exact)


def test_two_operators_on_two_streams():
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(6)
    streams, ops = [torch.cuda.Stream() for _ in range(2)], []
    gs = [torch.randn(2, 300, 400, generator=gen).cuda() for _ in range(2)]
    torch.cuda.synchronize()
    for s, g in zip(streams, gs):
        out = torch.empty((2, 300, 400), dtype=torch.bfloat16, device="cuda")
        ops.append((lm.Orthogonalize(g, out, stream=s), out))
    for _ in range(5):
        for op, _ in ops:
            op.forward()
    torch.cuda.synchronize()
    for g, (_, out) in zip(gs, ops):
        close(out, ref.ortho(g.double().cpu())[0])


@pytest.mark.parametrize("P,m,n", [(1, 100, 3000), (1, 3000, 130), (2, 300, 2050), (1, 16, 8192), (3, 129, 1600)])
def test_shared_contractions(P, m, n):
    """Few tiles and many columns: several blocks share a tile's contraction, and the last one adds the parts up in order; twice the same
    bits."""
    from paper_1905_10395_b200 import lm
    op, out = run(P, m, n, seed=n)
    first = out.view.clone()
    for _ in range(3):
        op.forward()
    torch.cuda.synchronize()
    assert torch.equal(out.view, first)
