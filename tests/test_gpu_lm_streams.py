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
