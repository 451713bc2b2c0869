"""GPU check of block-boundary norms whose rows are shared: inputs that repeat rows."""
import pytest
import torch

from tests import _lm_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 40), (3, 17)])
@pytest.mark.parametrize("D", [64, 75])
def test_one_row_for_all_without_a_block_output(shape, D):
    """Without y the forward pass writes only h, so `out`, the backward pass's x, may repeat rows like any input.  fp32 with a few
    roundings of values below 10: 2^-18 of them."""
    from paper_1905_10395_b200 import lm
    P, T = shape
    gen = torch.Generator().manual_seed(1)
    row, w = torch.randn(D, generator=gen), torch.randn(P, D, generator=gen)
    d_h = torch.randn(P, T, D, generator=gen)
    x = row.cuda().expand(P, T, D)
    h, dx = (torch.empty(P, T, D, device="cuda") for _ in range(2))
    dw = torch.empty(P, D, device="cuda")
    op = lm.BlockNorm(x=x, out=x, h=h, w_pre=w.cuda(), d_h=d_h.cuda(), dx=dx, dw_pre=dw)
    op.forward()
    op.backward()
    torch.cuda.synchronize()
    x64 = row.double().expand(P, T, D)
    want = ref.blocknorm_forward(x64, w_pre=w.double())[1]
    assert ((h.cpu().double() - want).abs() <= 2.0 ** -18 * 10).all()
    got, size = ref.blocknorm_backward(None, d_h.double(), x64, w_pre=w.double())
    assert ((dx.cpu().double() - got["dx"]).abs() <= 2.0 ** -18 * 30).all()
    assert ((dw.cpu().double() - got["dw_pre"]).abs() <= 2.0 ** -18 * size["dw_pre"] + 1e-6).all()
