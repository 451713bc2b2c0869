"""The convolution, the scan and the orthogonalised updates as they are used together: the example population whose blocks mix
tokens by a scan, against automatic differentiation of the same model and the 64-bit restatement of the updates."""
import pytest
import torch

from tests import _lm_mixer_reference as ref

pytestmark = pytest.mark.gpu


def _model(pop, p, tok, target):
    """Worker p's model in fp32 autograd, from the bf16 copies that the products read."""
    from paper_1905_10395_b200.lm_population import STATES as N
    F = pop.F
    f = lambda buf, n: pop._view(buf, n)[p].detach().float()  # noqa: E731
    q = {}
    for name, *_ in pop.segs:
        product = name == "table" or name.startswith(("w_in", "w_x", "w_out"))
        q[name] = f(pop.copy if product else pop.x, name).clone().requires_grad_()
    table = f(pop.x, "table").clone().requires_grad_()
    norm = lambda z: z * torch.rsqrt(z.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    silu = torch.nn.functional.silu
    x = table[tok] * pop.D ** 0.5
    h = norm(x) * q["w_pre0"]
    for i in range(pop.L):
        vz = h @ q[f"w_in{i}"].T
        v, z = vz[:, :F], vz[:, F:]
        taps = q[f"taps{i}"]
        padded = torch.cat([torch.zeros_like(v[:3]), v])
        v = silu(sum(padded[j:j + len(v)] * taps[:, j] for j in range(4)) + q[f"b_taps{i}"])
        dbc = v @ q[f"w_x{i}"].T
        delta = torch.nn.functional.softplus(dbc[:, :F] + q[f"dt_bias{i}"])
        B, C, A = dbc[:, F:F + N], dbc[:, F + N:], -torch.exp(q[f"a_log{i}"])
        s, ys = torch.zeros_like(A), []
        for t in range(len(v)):
            s = torch.exp(delta[t][:, None] * A) * s + (delta[t] * v[t])[:, None] * B[t]
            ys.append(s @ C[t])
        y = (torch.stack(ys) + q[f"skip{i}"] * v) * silu(z)
        y = y @ q[f"w_out{i}"].T
        x = x + torch.sigmoid(q[f"gate{i}"]) * norm(y) * q[f"w_post{i}"]
        h = norm(x) * q[f"w_pre{i + 1}"]
    loss = torch.nn.functional.cross_entropy(h @ q["table"].T, target)
    loss.backward()
    grads = {n: t.grad for n, t in q.items()}
    grads["table"] = grads["table"] + table.grad
    return loss.item(), grads


def test_gradients_of_the_whole_model():
    """bf16 activations and operands: every rounding is within 2^-8, a chain of L = 2 blocks has about sixteen of them on a path, and
    they are independent: 10 % of a tensor's gradient norm is far above what they leave (4 2^-8 = 1.6 %, and that twice where a
    gradient is the difference of two such terms), and far below a wrong term."""
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    pop = LmPopulation(3, 1, V=96, D=40, F=64, L=2, T=60, seed=4, mixer="scan")
    tok, target = (t.cuda() for t in markov_tokens(3, 60, 96, torch.Generator().manual_seed(5)))
    loss = pop.forward(tok, target)
    pop.backward()
    torch.cuda.synchronize()
    for p in range(3):
        want, grads = _model(pop, p, tok[p], target[p])
        assert abs(loss[p].item() - want) <= 2e-2 * abs(want)
        for name, g in grads.items():
            mine = pop._view(pop.g, name)[p]
            assert (mine - g).norm() <= 0.1 * g.norm() + 1e-6, (p, name, ((mine - g).norm() / g.norm()).item())
    pop.close()


@pytest.mark.parametrize("mixer", ["shift", "scan"])
def test_orthogonalised_step(mixer):
    """One step: the matrices move along their orthogonalised momentum (bounds as for the operator alone), the rest by AdamW as
    without it, and the bf16 copies follow."""
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    tok, target = (t.cuda() for t in markov_tokens(4, 64, 64, torch.Generator().manual_seed(8)))
    args = dict(V=64, D=32, F=64, L=2, T=64, tau=100, state="f32", seed=6, mixer=mixer)
    pop, plain = LmPopulation(4, 2, optimizer="ortho", **args), LmPopulation(4, 2, **args)
    before = pop.x.clone()
    assert torch.equal(before, plain.x)
    for q in (pop, plain):
        q.step(tok, target)
    torch.cuda.synchronize()
    assert torch.equal(pop.g, plain.g)
    moved = 0
    for name, shape, _, decayed in pop.segs:
        now, old = pop._view(pop.x, name), pop._view(before, name)
        assert torch.equal(pop._view(pop.copy, name), now.to(torch.bfloat16)), name
        if not decayed or name == "table":
            assert torch.equal(now, plain._view(plain.x, name)), name
            continue
        moved += 1
        g = pop._view(pop.g, name).double().cpu()
        out, momentum = ref.ortho(g, torch.zeros_like(g), scale=0.2 * max(shape) ** 0.5)
        step = (old.double() * (1 - pop.lr_ortho * 0.1) - now.double()).cpu() / pop.lr_ortho
        for p in range(4):
            assert (step[p] - out[p]).norm() <= 2.0 ** -6.5 * out[p].norm(), (name, p)
        # the gradient is stored in fp32: the momentum is its sum with zero
        assert torch.equal(pop._view(pop.momentum, name).double().cpu(), momentum)
    assert moved == (3 if mixer == "scan" else 2) * 2
    pop.close()
    plain.close()


@pytest.mark.parametrize("optimizer", ["adamw", "ortho"])
def test_training_runs_with_leaders(optimizer):
    """Twelve steps with pulls: everything stays finite, and the copies are the parameters' after every pull."""
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    pop = LmPopulation(4, 2, V=64, D=32, F=64, L=1, T=128, tau=4, seed=3, mixer="scan", optimizer=optimizer)
    gen = torch.Generator().manual_seed(7)
    for _ in range(12):
        tok, target = markov_tokens(4, 128, 64, gen)
        loss = pop.step(tok.cuda(), target.cuda())
        assert torch.isfinite(loss).all()
        if pop.t % pop.tau == 0:
            assert torch.equal(pop.copy, pop.x.to(torch.bfloat16))
    assert torch.isfinite(pop.x).all()
    pop.close()
