"""GPU check of the order between the language-model operators' own buffers and the streams they run on."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BUSY = 50_000_000            # clock cycles that a stream is kept busy for: about 25 ms


def test_the_table_of_tensors_is_copied_on_the_steps_stream():
    """The upload of the table and counter is work of the handle's stream: creation has drained that stream, a non-blocking one
    too, so no step can run ahead of it."""
    from paper_1905_10395_b200 import lm
    x, g = torch.ones(5000, device="cuda"), torch.ones(5000, device="cuda")
    state = {k: torch.zeros(5120, device="cuda") for k in ("m", "v")}
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    assert not s.query()
    opt = lm.AdamW([x], [g], stream=s, **state)
    assert s.query()
    opt.step(1e-2)
    torch.cuda.synchronize()
    assert opt.t() == 1 and torch.allclose(x, torch.full_like(x, 0.99), atol=1e-6)


@pytest.mark.parametrize("given", [False, True])
def test_the_readout_buffers_are_the_steps_streams(given):
    """moments() called first under another, busy stream: its buffers come from the pool of the stream that writes them, not from a
    block that the busy stream has freed and is still to use."""
    from paper_1905_10395_b200 import lm
    n = 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, g = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda")
    busy = torch.cuda.Stream()
    opt = lm.AdamW([x], [g], state="8bit", stream=torch.cuda.Stream() if given else None)
    opt.step(1e-2)
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        torch.cuda._sleep(BUSY)
        block = torch.empty(opt.values, device="cuda").zero_()          # still to be cleared when its memory is given back
        freed = block.data_ptr()
        del block
        m, v = opt.moments()
    assert freed not in (m.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    assert torch.isfinite(m).all() and (m != 0).any() and (v > 0).any()
    assert [t.data_ptr() for t in opt.moments()] == [m.data_ptr(), v.data_ptr()]


def test_the_population_steps_under_any_stream():
    """A population built under one stream and stepped under another, busy ones: the same bits as one that is alone."""
    from paper_1905_10395_b200.lm_population import LmPopulation, markov_tokens
    make = lambda: LmPopulation(3, 1, V=64, D=32, F=64, L=2, T=128, tau=2, seed=3)  # noqa: E731
    gen = torch.Generator().manual_seed(4)
    batches = [markov_tokens(3, 128, 64, gen) for _ in range(4)]
    alone = make()
    want = [alone.step(a.cuda(), b.cuda()).cpu() for a, b in batches]
    torch.cuda.synchronize()
    pop, s = make(), torch.cuda.Stream()
    got = []
    for a, b in batches:
        torch.cuda._sleep(BUSY // 10)
        with torch.cuda.stream(s):
            torch.cuda._sleep(BUSY // 10)
            loss = pop.step(a.cuda(), b.cuda())
            got.append(loss.clone())
    torch.cuda.synchronize()
    assert all(torch.equal(u, v.cpu()) for u, v in zip(want, got))
    assert torch.equal(pop.x, alone.x) and torch.equal(pop.copy, alone.copy)
    for q in (pop, alone):
        q.close()
