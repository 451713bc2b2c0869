"""The convolution, the scan and the orthogonalisation at the ends of their types' ranges: activations of far negative values."""
import pytest
import torch

from tests import _lm_mixer_reference as ref

pytestmark = pytest.mark.gpu

FAR = [-3e38, -1e38, -1e37, -1e35, -1e30, -1e5, -200.0, -104.0, -89.0, -88.5, -88.0, -87.5, -87.0, -60.0, 60.0, 88.0, 1e5, 1e38]
# silu and its slope at v: the exponent v log2(e) (|.| < 128 where the result is not zero) is rounded twice, by 2^-18 each, so
# the exponential is off by 2^-17.5, with the rest of the chain by less than 2^-16 of the magnitudes; sigmoids below 2^-126 count as
# zero, which |v| < 90 makes at most 90 2^-126 of the result
REL, FLOOR = 2.0 ** -16, 90 * 2.0 ** -126


def _near(got, want, size, half):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    bound = REL * size + half * want.abs() + FLOOR
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max().item()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_convolution_of_far_values(dtype):
    """pre sigmoid(pre) of pre = -1e38 is zero, and so is its slope; one tap of 1, so pre is x."""
    from paper_1905_10395_b200 import lm
    x = torch.tensor(FAR).to(dtype).repeat_interleave(4).view(1, len(FAR), 4)
    dev, w = x.cuda(), torch.ones((1, 4, 1), device="cuda")
    out, dx, dw, single = torch.empty_like(dev), torch.empty_like(dev), torch.empty_like(w), torch.empty_like(dev)
    op = lm.CausalConv(dev, w, out=out, d_out=torch.ones_like(dev), dx=dx, dw=dw)
    op.forward()
    op.backward()
    lm.CausalConv(dev, w, out=single, sequences=len(FAR)).forward()
    torch.cuda.synchronize()
    v = x.double()
    sg, half = torch.sigmoid(v), 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    _near(out, v * sg, (v * sg).abs(), half)
    _near(single, v * sg, (v * sg).abs(), half)
    _near(dx, sg * (1 + v * (1 - sg)), sg * (1 + v.abs() * (1 - sg)), half)


@pytest.mark.parametrize("T,S", [(1, 1), (24, 1), (24, 24), (600, 1)])
def test_scan_gated_by_far_values(T, S):
    """The gate z sigmoid(z) of z = -1e38 closes; single tokens, one chain and rows that are split into chains."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(T + S)
    D, N = len(FAR), 4
    z = torch.tensor(FAR)[torch.stack([torch.randperm(D, generator=gen) for _ in range(T)])][None]
    # y is of the order of 1, whose product with 1e38 is within fp32
    host = {k: torch.rand((1, T, n), generator=gen) * 0.1 for k, n in (("x", D), ("dt", D), ("b", N), ("c", N))}
    a_log = torch.randn((1, D, N), generator=gen)
    up = torch.rand((1, T, D), generator=gen) + 0.5
    dev = {k: v.cuda() for k, v in host.items()}
    new = {k: torch.zeros_like(v) for k, v in dev.items()}
    out, d_z, d_a = torch.zeros_like(dev["x"]), torch.zeros_like(dev["x"]), torch.zeros_like(a_log, device="cuda")
    grads = {} if S > 1 else dict(d_out=up.cuda(), d_x=new["x"], d_dt=new["dt"], d_a_log=d_a, d_b=new["b"], d_c=new["c"], d_z=d_z)
    op = lm.SelectiveScan(dev["x"], dev["dt"], a_log.cuda(), dev["b"], dev["c"], z=z.cuda(), out=out, sequences=S, **grads)
    op.forward()
    if grads:
        op.backward()
    torch.cuda.synchronize()
    f = {k: v.double() for k, v in host.items()}
    got, size = ref.scan(f["x"], f["dt"], a_log.double(), f["b"], f["c"], z.double(), None, None, None, up.double(), ref.edges_of(1, T, S, None))
    more = 2 * (T + D + 64) * 2.0 ** -22 / REL + 1                       # the scan's own error (test_gpu_lm_scan.py), in units of REL
    _near(out, got["out"], more * size["out"], 0.0)
    if grads:
        _near(d_z, got["d_z"], more * size["d_z"], 0.0)


@pytest.mark.parametrize("m,n", [(60, 90), (90, 60), (200, 300)])
@pytest.mark.parametrize("size", [1e-43, 1e-40, 1e-37, 1e-34, 1e36, 5e37])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orthogonalisation_of_any_magnitude(m, n, size, dtype):
    """X = U / |U| where 1 / |U| leaves fp32's range (|U| of 1e-40 or 1e40), without eps: bounds of test_gpu_lm_ortho.py."""
    from tests.test_gpu_lm_ortho import run
    if dtype == torch.bfloat16 and size < 2.0 ** -133:
        pytest.skip("below the least bf16 value, 2^-133: zeros")
    run(2, m, n, dtype, size=size, eps=0.0, seed=m)


@pytest.mark.parametrize("first", [7.9, 5.0])
@pytest.mark.parametrize("m,n", [(1, 1), (2, 3), (130, 1), (1, 300)])
def test_orthogonalisation_up_to_the_stated_range(first, m, n):
    """The largest singular values in range, below 8, with a polynomial that brings them back.  A matrix of rank one, whose singular
    value is 1 to begin with: 7.8, then 7.8 (7.9 - 0.1 61) = 14, which is the last."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(m)
    g = torch.randn((1, m, 1), generator=gen) * torch.randn((1, 1, n), generator=gen)
    for steps, coefficients in ((1, (first, 0.0, 0.0)), (2, (first, -0.1, 0.0)), (3, (1.5, -0.5, 0.0)), (2, (first, 0.0, -0.01))):
        out = torch.empty((1, m, n), dtype=torch.bfloat16, device="cuda")
        lm.Orthogonalize(g.cuda(), out, coefficients=coefficients, steps=steps).forward()
        torch.cuda.synchronize()
        want, _ = ref.ortho(g.double(), coefficients=coefficients, steps=steps)
        got = out.double().cpu()
        # X and G are off by 2^-11 of them at most, so v^2 by 2^-9.4 and v^4 by 2^-8.4 of them: at v = 7.9 the step's factor by
        # 0.1 62 2^-9.4 < 0.01 or 0.01 3900 2^-8.4 < 0.12, of a result whose factor is 1.7 or -31
        assert (got - want).norm() <= 2.0 ** -5 * max(want.norm(), first), (steps, coefficients, got.norm(), want.norm())
