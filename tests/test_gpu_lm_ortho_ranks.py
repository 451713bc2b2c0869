"""GPU check of the orthogonalised updates of matrices of few large singular values (a gradient of few tokens), against 64 bits.

Bounds.  A rounding to fp16 is off by 2^-12.3 of the norm of a matrix of values of any size (2^-10 / sqrt(12) of a value's power of
two), 2^-11.8 at most; where singular values are small or zero every later step multiplies it by a = 3.4445.  X_4 passes one more step, from a
norm of at most 1.8 times the result's (singular values that are not small lie in 0.68 .. 1.2): 1.8 3.4 2^-11.8 = 1.7e-3.  What the X in front
of it are rounded by is carried on: through Q up to 128 rows; else through its diagonal, which is a less 2.7 k / r for k equal singular
values of r, so that 0.79 k / r of it is not, on the 1 - k / r of all directions that are null.  From X_0 to X_3 that is amplified by 485, 141,
41 and 12, from norms of 1, 3.4, 11 (8.4) and 8 where k = 64, of a result's norm of 8: in the squares 96 0.79 (k / r) sqrt(1 - k / r)
2^-12.3, 5.3e-3 at k / r = 1/2 and less elsewhere.  With 2e-3 of G and Q (2 sqrt(15) 2^-12) and 1.7e-3 of the rounding to bf16: 6.2e-3 in the
squares, below 2^-7.  A matrix of full rank hides what falls on its few small singular values: the latter two, below 2^-8."""
import pytest
import torch

from tests import _lm_mixer_reference as ref

pytestmark = pytest.mark.gpu


def _off(P, m, n, rank, noise, dtype=torch.float32, seed=0):
    from paper_1905_10395_b200 import lm
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    g = (r(P, m, rank) @ r(P, rank, n) * rank ** -0.5 if rank else r(P, m, n)) + noise * r(P, m, n)
    g = (g * 1e-3).to(dtype)
    out = torch.empty((P, m, n), dtype=torch.bfloat16, device="cuda")
    lm.Orthogonalize(g, out).forward()
    want, _ = ref.ortho(g.double())
    norm = torch.linalg.matrix_norm
    return (norm(out.double() - want) / norm(want)).max().item()


# one block a matrix; launches of up to 128 rows and beyond, wide and tall
SIZES = [(8, 16, 16), (4, 64, 64), (2, 128, 128), (3, 100, 250), (2, 16, 2000), (1, 120, 700), (2, 300, 400), (1, 700, 900), (1, 800, 1024), (2, 1024, 1024), (1, 1000, 600), (1, 1500, 1100)]


@pytest.mark.parametrize("P,m,n", SIZES)
@pytest.mark.parametrize("rank", [1, 4, 16, 64])
@pytest.mark.parametrize("noise", [0.0, 1e-3])
def test_few_large_singular_values(P, m, n, rank, noise):
    off = _off(P, m, n, min(rank, min(m, n)), noise, seed=rank)
    assert off <= 2.0 ** -7, off


@pytest.mark.parametrize("P,m,n", SIZES)
def test_all_singular_values(P, m, n):
    off = _off(P, m, n, 0, 0.0)
    assert off <= 2.0 ** -8, off


@pytest.mark.parametrize("rank", [1, 16])
def test_gradients_in_bf16(rank):
    off = _off(2, 512, 640, rank, 1e-3, torch.bfloat16)
    assert off <= 2.0 ** -7, off
