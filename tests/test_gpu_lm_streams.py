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
