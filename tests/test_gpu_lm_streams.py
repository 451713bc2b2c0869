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


def _bound(stream=None):
    from paper_1905_10395_b200 import lm
    gen = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    table, d_table, rows = mk(1, 40, 64), torch.zeros(1, 40, 64, device="cuda"), [mk(1, 30, 64) for _ in range(6)]
    tok = torch.randint(0, 40, (1, 30), generator=gen, device="cuda")
    e = lm.Embedding(tok, table=table, out=rows[0], d_out=rows[1], d_table=d_table, stream=stream)
    n = lm.BlockNorm(x=rows[0], out=rows[0], h=rows[2], w_pre=mk(1, 64), d_out=rows[3], d_h=rows[4], dx=rows[5], stream=stream)
    p = mk(1000)
    a = lm.AdamW([p], [mk(1000)], state="8bit", stream=stream)
    a.step(1e-2)
    a.moments()
    torch.cuda.synchronize()
    return e, n, a, (rows, d_table, p)


def test_a_call_is_not_left_out_of_a_capture():
    """Operators of the default stream under a capture of another: refused, nothing is launched, and the capture goes on."""
    from paper_1905_10395_b200 import api
    e, n, a, (rows, d_table, p) = _bound()
    before = [t.clone() for t in (*rows, d_table, p)]
    graph, count = torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        count += 1
        for call in (e.forward, e.backward, n.forward, n.backward, lambda: a.step(1e-2), a.moments, lambda: a.set_step(3)):
            with pytest.raises(api.LsgdError) as err:
                call()
            assert err.value.status == api.ERR_STATE
        count += 1
    graph.replay()
    torch.cuda.synchronize()
    assert count.item() == 2 and a.t() == 1
    assert all(torch.equal(u, v) for u, v in zip(before, (*rows, d_table, p)))


def test_a_stream_that_the_capture_has_been_forked_to():
    """The operators' stream joins the capture through an event: their calls are captured, whatever stream is current."""
    side = torch.cuda.Stream()
    e, n, a, (rows, d_table, p) = _bound(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        e.forward()
        n.forward()
        a.step(1e-2)
        torch.cuda.current_stream().wait_stream(side)
    x = p.clone()
    rows[0].zero_()
    rows[2].zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(p, x) and a.t() == 4
    assert (rows[0].abs().sum(-1) > 0).all() and (rows[2].abs().sum(-1) > 0).all()
