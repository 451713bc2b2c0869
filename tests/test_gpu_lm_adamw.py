"""GPU check of the AdamW step over many tensors (lsgd_adamw_*).

The moments are defined operation by operation in fp32 (include/lsgd.h), so a restatement on the CPU in fp32 gives their bits,
codes and scales of the 8-bit ones included.  The parameters' step is checked in 64 bits: x loses at most half a unit for the
product with 1 - lr wd, half a unit for the sum, and 2^-20 of the step itself (approximate square root and reciprocal, each
within 2^-22, and four roundings)."""
import numpy as np
import pytest
import torch

from tests import _lm_reference as ref

pytestmark = pytest.mark.gpu

B = 256
U32 = 0xFFFFFFFF
B1, B2, EPS = 0.9, 0.95, 1e-8


def mix(h):
    h = (h * 0x9E3779B1) & U32
    h = h ^ (h >> 15)
    h = (h * 0x85EBCA77) & U32
    return h ^ (h >> 13)


def decode(code, scale, signed):
    """Codes as the header defines them, from their fields, in fp32 (every value times its scale is one rounding)."""
    c = code.to(torch.int64)
    lead, bias, bits = (c & 127, 15, 112) if signed else (c, 31, 96)
    e, f = lead >> 3, (lead & 7).double()
    v = torch.where(e == 0, f / 8 * 2.0 ** (1 - bias), (1 + f / 8) * torch.exp2(e.double() - bias))
    v = torch.where(c > 127, -v, v) if signed else v
    return v.float() * scale.float()[:, None]


def encode(z, rnd16, signed):
    top = z.abs().amax(1)
    scale = torch.where(top < 2.0 ** -100, torch.zeros_like(top), top * torch.tensor(0.53333336))
    inv = torch.where(scale > 0, 1 / scale, torch.zeros_like(scale))
    small = torch.tensor(2.0 ** (-112 if signed else -96))
    folded = z.abs() * (inv * small)[:, None]
    plain = (z.abs() * inv[:, None]) * small
    q = torch.where(scale[:, None] < 16384, folded, plain)
    bits = q.contiguous().view(torch.int32).long()
    code = (bits + (rnd16 << 4)) >> 20
    if signed:
        code = code + 128 * (z < 0)
    else:
        code = torch.where((bits > 0) & (bits < 1 << 20), torch.ones_like(code), code)
    return code, scale


class Model:
    """The whole state on the CPU, every tensor's moments begun at a multiple of 256."""

    def __init__(self, sizes, params, wd, state, seed, t=0):
        self.sizes, self.wd, self.state, self.seed, self.t = sizes, wd, state, seed, t
        self.x = [p.clone() for p in params]
        self.starts = np.cumsum([0] + [(n + B - 1) // B * B for n in sizes])
        n = int(self.starts[-1])
        self.m, self.v = torch.zeros(n), torch.zeros(n)
        self.cm, self.cv = torch.zeros(n, dtype=torch.int64), torch.zeros(n, dtype=torch.int64)
        self.sm, self.sv = torch.zeros(n // B), torch.zeros(n // B)

    def step(self, grads, lr, gs=None):
        self.t += 1
        n = len(self.m)
        if self.state == "8bit":
            self.m = decode(self.cm.view(-1, B), self.sm, True).view(-1)
            self.v = decode(self.cv.view(-1, B), self.sv, False).view(-1)
        g = torch.zeros(n)
        for s, k, gr in zip(self.starts, self.sizes, grads):
            g[s:s + k] = gr.float() if gs is None else gr.float() * torch.tensor(gs)
        f = lambda v: torch.tensor(v, dtype=torch.float64).float()  # noqa: E731
        m = self.m * f(B1) + g * f(1 - B1)
        v = self.v * f(B2) + g * f(1 - B2) * g
        self.bound = []
        for i, (s, k) in enumerate(zip(self.starts, self.sizes)):
            x = self.x[i].double()
            step = lr * (m[s:s + k].double() / (1 - B1 ** self.t)) / (torch.sqrt(v[s:s + k].double() / (1 - B2 ** self.t)) + EPS)
            self.x[i] = x * (1 - lr * float(np.float32(self.wd[i]))) - step
            self.bound.append(2.0 ** -23 * (x.abs() + step.abs()) + 2.0 ** -20 * step.abs() + 1e-37)
        if self.state == "8bit":
            h = mix(torch.arange(n) ^ mix(mix(self.seed) ^ self.t)).view(-1, B)
            self.cm, self.sm = encode(m.view(-1, B), h & 0xFFFF, True)
            self.cv, self.sv = encode(v.view(-1, B), h >> 16, False)
            self.m, self.v = decode(self.cm, self.sm, True).view(-1), decode(self.cv, self.sv, False).view(-1)
            self.cm, self.cv = self.cm.view(-1), self.cv.view(-1)
        else:
            self.m, self.v = m, v


def build(sizes, state="f32", grad="f32", copies=True, offset=0, seed=0, wd=None, scale=1.0, t=0, stream=None):
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(seed)
    gd = {"f32": torch.float32, "bf16": torch.bfloat16}[grad]
    host = [torch.randn(n, generator=gen) for n in sizes]
    wd = [0.1 * (i % 3) for i in range(len(sizes))] if wd is None else wd
    p = [ref.Guarded((n,), (1,), torch.float32, offset, h) for n, h in zip(sizes, host)]
    g = [ref.Guarded((n,), (1,), gd, offset, torch.randn(n, generator=gen).mul_(scale).to(gd)) for n in sizes]
    c = [ref.Guarded((n,), (1,), torch.bfloat16, offset) for n in sizes] if copies else None
    opt = lm.AdamW([a.view for a in p], [a.view for a in g], state=state, copies=[a.view for a in c] if c else None, beta1=B1, beta2=B2,
                   eps=EPS, weight_decay=wd, seed=seed + 77, step=t, stream=stream)
    return opt, Model(sizes, host, wd, state, seed + 77, t), p, g, c, gen


def check(opt, model, p, g, c):
    torch.cuda.synchronize()
    m, v = opt.moments()
    torch.cuda.synchronize()
    m, v = m.cpu(), v.cpu()
    for i, (s, k) in enumerate(zip(model.starts, model.sizes)):
        got = p[i].view.cpu()
        assert ((got.double() - model.x[i]).abs() <= model.bound[i]).all(), (i, k)
        model.x[i] = got.clone()                                   # errors do not pile up from step to step
        assert torch.equal(m[s:s + k], model.m[s:s + k]) and torch.equal(v[s:s + k], model.v[s:s + k]), (i, k)
        if c:
            assert torch.equal(c[i].view.cpu(), got.to(torch.bfloat16))
        if opt.state == "8bit":
            e = (k + B - 1) // B * B
            assert torch.equal(opt.m[s:s + e].cpu().long() & 127, model.cm[s:s + e] & 127)
            assert torch.equal(opt.v[s:s + e].cpu().long(), model.cv[s:s + e])
            assert torch.equal(opt.m_scale[s // B:(s + e) // B].cpu(), model.sm[s // B:(s + e) // B])
            assert torch.equal(opt.v_scale[s // B:(s + e) // B].cpu(), model.sv[s // B:(s + e) // B])
    for b in p + g + (c or []):
        assert b.intact()


SIZES = [1, 2, 7, 8, 9, 255, 256, 257, 0, 1000, 4095, 4096, 4097, 8200, 20000]


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("copies", [True, False])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_steps(state, grad, copies, offset):
    opt, model, p, g, c, gen = build(SIZES, state, grad, copies, offset, seed=offset)
    for k in range(4):
        for b in g:
            b.view.copy_(torch.randn(b.view.shape, generator=gen).mul_(10.0 ** (k - 2)))
        opt.step(1e-2)
        model.step([b.view.cpu() for b in g], 1e-2)
        check(opt, model, p, g, c)
    assert opt.t() == 4


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_many_tensors_and_large_ones(state):
    """More tensors than blocks of the grid, and one with more chunks than the grid."""
    for sizes in ([37 + i for i in range(1500)], [148 * 4 * 4096 * 2 + 333]):
        opt, model, p, g, c, gen = build(sizes, state, "bf16", True, 0, seed=3)
        opt.step(1e-3)
        model.step([b.view.cpu() for b in g], 1e-3)
        check(opt, model, p, g, c)


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-16, 1e-6, 1e6, 1e12])
def test_sizes_of_gradients(state, scale):
    """Zero gradients and states, blocks below the smallest scale, and scales past the folded powers of two."""
    opt, model, p, g, c, gen = build([3000, 5], state, "f32", False, 0, seed=5, scale=scale)
    for _ in range(3):
        opt.step(1e-2)
        model.step([b.view.cpu() for b in g], 1e-2)
        check(opt, model, p, g, c)
    assert all(torch.isfinite(b.view).all() for b in p)


def test_restored_step_and_gradient_scale():
    opt, model, p, g, c, gen = build([5000, 77], "8bit", "bf16", True, 0, seed=6, t=1000)
    assert opt.t() == 1000
    gs = torch.tensor([0.25], device="cuda")
    for k in range(2):
        opt.step(1e-3, grad_scale=gs)
        model.step([b.view.cpu() for b in g], 1e-3, gs=0.25)
        check(opt, model, p, g, c)
    opt.set_step(7)
    model.t = 7
    opt.step(1e-3)
    model.step([b.view.cpu() for b in g], 1e-3)
    check(opt, model, p, g, c)
    assert opt.t() == 8


def test_state_given_by_the_caller_continues():
    """A run of four steps is the run of two, its buffers and counter given to a new handle, and two more."""
    from paper_1905_10395_b200 import lm
    for state in ("f32", "8bit"):
        opt, _, p, g, c, _ = build([3001, 10], state, "f32", False, seed=8)
        other, _, q, h, _, _ = build([3001, 10], state, "f32", False, seed=8)
        for _ in range(4):
            opt.step(1e-2)
        for _ in range(2):
            other.step(1e-2)
        again = lm.AdamW([b.view for b in q], [b.view for b in h], m=other.m, v=other.v, m_scale=other.m_scale, v_scale=other.v_scale,
                         beta1=B1, beta2=B2, eps=EPS, weight_decay=[0.0, 0.1], seed=8 + 77, step=other.t())
        for _ in range(2):
            again.step(1e-2)
        torch.cuda.synchronize()
        assert all(torch.equal(a.view, b.view) for a, b in zip(p, q))


def test_rounding_has_the_right_mean():
    """Moments that change by less than a code's spacing move all the same: after 64 steps of a constant gradient from zero, v is
    near (1 - beta2^64) g^2 on average, with the scatter of rounded steps (spacing 1/8, 2^16 values: a mean within 1%)."""
    n = 1 << 16
    opt, _, p, g, _, _ = build([n], "8bit", "f32", False, seed=9)
    gr = torch.linspace(0.5, 1.0, n).double()
    g[0].view.copy_(gr)
    for _ in range(64):
        opt.step(1e-3)
    m, v = opt.moments()
    torch.cuda.synchronize()
    assert abs(float((m.cpu().double() / ((1 - B1 ** 64) * gr)).mean()) - 1) < 0.01
    assert abs(float((v.cpu().double() / ((1 - B2 ** 64) * gr * gr)).mean()) - 1) < 0.01


def test_not_finite_gradients():
    """fp32 moments: the value alone is lost.  8 bits: its block of 256 reads as NaN, every other block is what it was."""
    for bad in (float("nan"), float("inf")):
        for state in ("f32", "8bit"):
            res = []
            for poison in (False, True):
                opt, _, p, g, _, _ = build([1000], state, "f32", False, seed=10)
                if poison:
                    g[0].view[300] = bad
                opt.step(1e-2)
                m, v = opt.moments()
                torch.cuda.synchronize()
                res.append([t.clone().cpu() for t in (p[0].view, m[:1000], v[:1000])])
            lost = torch.zeros(1000, dtype=torch.bool)
            lost[300] = True
            assert torch.equal(res[0][0][~lost], res[1][0][~lost]) and not torch.isfinite(res[1][1][300])
            if state == "8bit":
                lost[256:512] = True
                assert torch.isnan(res[1][1][256:512]).all() and torch.isnan(res[1][2][256:512]).all()
            for a, b in zip(res[0][1:], res[1][1:]):
                assert torch.equal(a[~lost], b[~lost])


def test_captured_in_a_graph():
    """The counter is on the device: a replayed step is the next step."""
    s = torch.cuda.Stream()
    a, _, p, g, _, _ = build([5000, 300], "8bit", "f32", False, seed=11, stream=s)
    b, _, q, h, _, _ = build([5000, 300], "8bit", "f32", False, seed=11)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a.step(1e-2)
        a.step(1e-2)
    for _ in range(3):
        graph.replay()
    for _ in range(6):
        b.step(1e-2)
    torch.cuda.synchronize()
    assert a.t() == b.t() == 6
    assert all(torch.equal(x.view, y.view) for x, y in zip(p, q)) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v)


def test_moments_of_its_own_on_another_stream():
    """Moments that the binding allocates are cleared on the step's stream: no order with the current one is needed for them."""
    from paper_1905_10395_b200 import lm
    n = 1 << 22
    gen = torch.Generator(device="cuda").manual_seed(12)
    p, g = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda")
    got = []
    for stream in (None, torch.cuda.Stream()):
        x = p.clone()
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)                 # the current stream is busy for about 10 ms
        opt = lm.AdamW([x], [g], state="8bit", stream=stream)
        for _ in range(2):
            opt.step(1e-2)
        torch.cuda.synchronize()
        got.append((x, opt.m.clone(), opt.v.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got))
