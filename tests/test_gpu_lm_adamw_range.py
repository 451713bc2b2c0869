"""GPU check of the AdamW step at the ends of its range: moments of very different sizes in one block, tiny and infinite ones, and an
eps that does not hide them."""
import pytest
import torch

from tests import test_gpu_lm_adamw as base

pytestmark = pytest.mark.gpu

B = base.B


def encode_by_contract(z, rnd16, signed):
    """As the header has it: a second moment above zero has a code above zero, however small it is in its block."""
    code, scale = base_encode(z, rnd16, signed)
    if not signed:
        code = torch.where((z > 0) & (scale > 0)[:, None], code.clamp(min=1), code)
    return code, scale


base_encode = base.encode


def test_small_second_moments_beside_a_large_one(monkeypatch):
    """One gradient of 1 in every block, the others 2^-28, for 30 steps: v of the others is 2^-56 of the block's.

    Their bound.  From the second step on a stored m is at most its smallest code, 2^-17 scale, and a stored v at least its
    smallest, 2^-33 scale, with scale = (1 - b^t) / 1.875 for a largest gradient of 1.  So the step is at most
    0.9 2^-17 / 1.875 / sqrt(0.95 2^-33 / 1.875) = 0.477 lr, and less at small t (m's factor (1 - b1^(t-1)) / (1 - b1^t) is the
    smaller one); the first is 2^-28 / (2^-28 + 1e-8) = 0.27 lr."""
    monkeypatch.setattr(base, "encode", encode_by_contract)
    n = 64 * B
    opt, model, p, g, c, _ = base.build([n], "8bit", "f32", False, seed=21, wd=[0.0])
    gr = torch.full((n,), 2.0 ** -28)
    gr[::B] = 1.0
    g[0].view.copy_(gr)
    small = gr < 1
    last = p[0].view.cpu().clone()
    p[0].view.zero_()
    model.x[0] = torch.zeros(n)
    last.zero_()
    for _ in range(30):
        opt.step(1.0)
        model.step([gr], 1.0)
        base.check(opt, model, p, g, c)
        now = p[0].view.cpu()
        step = (now - last).abs()
        last = now.clone()
        assert step[small].max() <= 0.48 and 0.8 <= step[~small].min() and step[~small].max() <= 1.2
        assert (opt.v.cpu() > 0).all()
        p[0].view.zero_()
        model.x[0].zero_()
        last.zero_()


def test_far_apart_values_keep_their_codes(monkeypatch):
    """Gradients over 40 binades in every block, fresh ones every step: codes, scales, moments and parameters."""
    monkeypatch.setattr(base, "encode", encode_by_contract)
    opt, model, p, g, c, gen = base.build([5000, 300], "8bit", "f32", False, seed=22)
    for _ in range(4):
        for b in g:
            b.view.copy_(torch.randn(b.view.shape, generator=gen) * torch.exp2(-40 * torch.rand(b.view.shape, generator=gen)))
        opt.step(1e-2)
        model.step([b.view.cpu() for b in g], 1e-2)
        base.check(opt, model, p, g, c)


@pytest.mark.parametrize("moment", ["m", "v"])
def test_an_infinity_whose_rounding_adds_nothing(moment):
    """A block with an infinite moment reads as NaN whatever random bits its values get: here those of the infinity are 0."""
    n, seed = 1 << 18, 23
    h = base.mix(torch.arange(n) ^ base.mix(base.mix(seed + 77) ^ 1))
    at = int(torch.nonzero((h & 0xFFFF if moment == "m" else h >> 16) == 0)[0])
    opt, _, p, g, _, _ = base.build([n], "8bit", "f32", False, seed=seed)
    g[0].view[at] = float("inf")
    opt.step(1e-2)
    m, v = opt.moments()
    torch.cuda.synchronize()
    lost = torch.zeros(n, dtype=torch.bool, device="cuda")
    lost[at // B * B:at // B * B + B] = True
    for t in (m, v):
        assert torch.isnan(t[lost]).all() and torch.isfinite(t[~lost]).all()


@pytest.mark.parametrize("size", [1e-14, 4e-15, 1e-15, 1e-20])
def test_blocks_below_the_least_scale(size):
    """Blocks whose second moments are stored as zeros, at the least eps: m^ is at most 2^-50 / sqrt(1 - b2) there, so a step is at
    most lr / sqrt(1 - b2).  A gradient of 1e-14 keeps its v: m^ / sqrt(v^) = 1, and a code of v is within a factor of 9 / 8."""
    from paper_1905_10395_b200 import lm
    x, g = torch.zeros(B, device="cuda"), torch.full((B,), size, device="cuda")
    opt = lm.AdamW([x], [g], state="8bit", beta1=base.B1, beta2=base.B2, eps=2.0 ** -50)
    bound = 9 / 8 if size == 1e-14 else (1 - base.B2) ** -0.5
    for _ in range(40):
        x.zero_()
        opt.step(1.0)
        assert 0 <= float(-x.max()) and float(x.abs().max()) <= bound * 1.001


@pytest.mark.parametrize("eps", [1.2e-38, 1e-30, 1e-20, 1e-16, 1e-13, 1e-11, 1e-8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_roots_of_small_second_moments(eps, grad):
    """fp32 moments down to subnormal ones, against the step of the moments as they are stored: 2^-20 of it, as in the other tests
    (approximate root and reciprocal, within 2^-22 each, and four roundings).  Sizes from 1 to 1e-21, tensors off 32 bytes too."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator(device="cuda").manual_seed(24)
    n, dtype = 6000, {"f32": torch.float32, "bf16": torch.bfloat16}[grad]
    for offset in (0, 1):
        buf = [torch.zeros(n + 1, device="cuda", dtype=t)[offset:offset + n] for t in (torch.float32, dtype)]
        x, g = buf
        sizes = torch.logspace(-21, 0, n, dtype=torch.float64, device="cuda")
        opt = lm.AdamW([x], [g], beta1=base.B1, beta2=base.B2, eps=eps)
        for t in range(1, 4):
            g.copy_(torch.randn(n, generator=gen, device="cuda").double() * sizes)
            x.zero_()
            opt.step(1.0)
            m, v = (z[:n].double() for z in opt.moments())
            want = (m / (1 - base.B1 ** t)) / (torch.sqrt(v / (1 - base.B2 ** t)) + eps)
            assert (((-x).double() - want).abs() <= 2.0 ** -20 * want.abs() + 1e-37).all(), (offset, t)


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("scale", [1e-25, 1e-16, 1e-12, 1.0, 1e12])
def test_steps_with_a_small_eps(state, scale, monkeypatch):
    """The whole step of every type at an eps whose kernels lift small roots."""
    monkeypatch.setattr(base, "EPS", 2.0 ** -50)
    for grad, offset in (("f32", 0), ("bf16", 1)):
        opt, model, p, g, c, gen = base.build([3000, 4096, 5], state, grad, True, offset, seed=25, scale=scale)
        for _ in range(3):
            opt.step(1e-2)
            model.step([b.view.cpu() for b in g], 1e-2)
            base.check(opt, model, p, g, c)
