"""The language-model operators as they are used together: the example population against automatic differentiation of the
same model, and its training with leaders."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _model(pop, p, tok, target):
    """Worker p's model in fp32 autograd, from the bf16 copies that the products read."""
    f = lambda buf, n: pop._view(buf, n)[p].detach().float()  # noqa: E731
    q = {}
    for name, *_ in pop.segs:
        product = name == "table" or name.startswith("w1") or name.startswith("w2")
        q[name] = f(pop.copy if product else pop.x, name).clone().requires_grad_()
    table = f(pop.x, "table").clone().requires_grad_()
    norm = lambda z: z * torch.rsqrt(z.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    x = table[tok] * pop.D ** 0.5
    h = norm(x) * q["w_pre0"]
    for i in range(pop.L):
        prev = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
        u = torch.relu(torch.cat([h, prev], 1) @ q[f"w1_{i}"].T + q[f"b1_{i}"])
        y = u @ q[f"w2_{i}"].T
        x = x + torch.sigmoid(q[f"gate{i}"]) * norm(y) * q[f"w_post{i}"]
        h = norm(x) * q[f"w_pre{i + 1}"]
    loss = torch.nn.functional.cross_entropy(h @ q["table"].T, target)
    loss.backward()
    grads = {n: t.grad for n, t in q.items()}
    grads["table"] = grads["table"] + table.grad
    return loss.item(), grads


def test_gradients_of_the_whole_model():
    """bf16 activations and operands: every rounding is within 2^-8, a chain of L = 2 blocks has about ten of them on a path, and
    they are independent: 10% of a tensor's gradient norm is far above what they leave, and far below a wrong term."""
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    pop = LmPopulation(3, 1, V=96, D=40, F=64, L=2, T=100, seed=4)
    tok, target = markov_tokens(3, 100, 96, torch.Generator().manual_seed(5))
    tok, target = tok.cuda(), target.cuda()
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


@pytest.mark.parametrize("state", ["8bit", "f32"])
def test_training_with_leaders(state):
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    pop = LmPopulation(4, 2, V=64, D=32, F=64, L=1, T=256, tau=5, state=state, seed=6)
    gen = torch.Generator().manual_seed(7)
    losses = []
    for t in range(80):
        tok, target = markov_tokens(4, 256, 64, gen)
        losses.append(pop.step(tok.cuda(), target.cuda()).cpu().numpy())
        if pop.t % pop.tau == 0:
            ll, gl = pop.lsgd.leaders()
            assert gl == int(np.argmin(losses[-1]))
            assert list(ll) == [int(np.argmin(losses[-1][:2])), 2 + int(np.argmin(losses[-1][2:]))]
            assert torch.equal(pop.copy, pop.x.to(torch.bfloat16))
    assert losses[0].mean() > 3.5 and losses[-1].mean() < 1.2, (losses[0], losses[-1])     # log 64 = 4.16; the source has 0.69
    assert pop.opt.t() == 80
    pop.close()


def test_a_population_without_blocks():
    """L = 0: the embedded tokens' norm and the output layer alone.  Nothing is read that no kernel has written (10 % of a tensor's
    gradient as in the other tests of whole models: bf16 operands)."""
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    pop = LmPopulation(2, 1, V=64, D=32, F=64, L=0, T=100, seed=4)
    for t in (*pop.res, *pop.d_res, *pop.h, *pop.d_h, pop.logits):
        t.fill_(float("nan"))
    tok, target = (t.cuda() for t in markov_tokens(2, 100, 64, torch.Generator().manual_seed(5)))
    loss = pop.forward(tok, target)
    pop.backward()
    torch.cuda.synchronize()
    for p in range(2):
        want, grads = _model(pop, p, tok[p], target[p])
        assert abs(loss[p].item() - want) <= 2e-2 * abs(want)
        for name, g in grads.items():
            mine = pop._view(pop.g, name)[p]
            assert (mine - g).norm() <= 0.1 * g.norm() + 1e-6, (p, name)
    pop.close()
