"""Host-only checks of what the convolution, the scan and the orthogonalisation refuse at the ends of their ranges.  No GPU."""
import ctypes as C

import pytest
import torch

from tests.test_lm_binding import Devices
from tests.test_lm_mixer_boundary import MB, _conv, _ortho, _refused, _scan, api, lm  # noqa: F401  (fixtures)


@pytest.fixture
def devices(monkeypatch, lm):  # noqa: F811
    return Devices(monkeypatch, lm)


def test_most_sequences(api):  # noqa: F811
    """As many sequences as rows may be, of all workers together: kernels index both, and the step behind the last, in 32 bits.  One less passes,
    to the refusal of the scratch's alignment."""
    L, most = api.lib(), (1 << 31) - (1 << 20)
    for make, calls in ((_conv, (L.lsgd_conv_forward, L.lsgd_conv_backward)), (_scan, (L.lsgd_scan_forward, L.lsgd_scan_backward))):
        for P, S in ((2, most // 2), (1, most), (1, (1 << 31) - 1)):
            for call in calls:
                assert call(C.byref(make(api, P=P, T=5, seq=api.Sequences(MB * 70, 0, S), scratch=8, scratch_bytes=1 << 60)), None) == 8, (P, S)
                assert call(C.byref(make(api, P=P, T=5, seq=api.Sequences(MB * 70, 0, most // P - 1), scratch=8, scratch_bytes=1 << 60)), None) == 3
                assert call(C.byref(make(api, P=P, T=0, seq=api.Sequences(None, 0, S))), None) == 8


def test_a_backward_pass_needs_saved_states_that_something_has_written(lm, devices, monkeypatch):  # noqa: F811
    """Without `out` the operator has no forward pass that would fill states of its own; with the caller's it has."""
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: real(*a, **k))
    x, a, bc = torch.zeros(2, 12, 8), torch.zeros(2, 8, 4), torch.zeros(2, 12, 4)
    new = lambda t: torch.zeros_like(t)  # noqa: E731
    grads = dict(d_out=new(x), d_x=new(x), d_dt=new(x), d_a_log=new(a), d_b=new(bc), d_c=new(bc))
    _refused(lm, lm.api.ERR_INVALID_ARG, lambda: lm.SelectiveScan(x, x, a, bc, bc, **grads))
    saved = torch.zeros(2, 2, 8, 4)
    assert lm.SelectiveScan(x, x, a, bc, bc, saved=saved, **grads).saved is saved
    assert lm.SelectiveScan(x, x, a, bc, bc, out=new(x), **grads).saved.shape == saved.shape
    # no rows: nothing is saved
    none = lambda t: torch.zeros(2, 0, t.shape[2])  # noqa: E731
    x, bc = none(x), none(bc)
    lm.SelectiveScan(x, x, a, bc, bc, d_out=new(x), d_x=new(x), d_dt=new(x), d_a_log=new(a), d_b=new(bc), d_c=new(bc))


class Sized:
    """A tensor's shape, type and strides, without its memory."""

    def __init__(self, *shape, dtype=torch.float32):
        self.t = torch.zeros(shape, dtype=dtype, device="meta")

    def __getattr__(self, name):
        return getattr(self.t, name)

    def data_ptr(self):
        return MB


@pytest.mark.parametrize("n", [(1 << 32) + 8, 1 << 31])
def test_sizes_of_more_than_32_bits_are_refused(lm, devices, n):  # noqa: F811
    """A size that the descriptor holds in 32 bits: not taken modulo 2^32, which would leave most of the output as it was."""
    s, bf = Sized, torch.bfloat16
    calls = [lambda: lm.CausalConv(s(1, 4, n), s(1, n, 2), out=s(1, 4, n)), lambda: lm.CausalConv(s(n, 4, 8), s(n, 8, 2), out=s(n, 4, 8)),
             lambda: lm.CausalConv(s(1, 4, 8), s(1, 8, n), out=s(1, 4, 8)),
             lambda: lm.CausalConv(s(1, 0, 8), s(1, 8, 2), out=s(1, 0, 8), sequences=n),
             lambda: lm.SelectiveScan(s(1, 4, n), s(1, 4, n), s(1, n, 2), s(1, 4, 2), s(1, 4, 2), out=s(1, 4, n)),
             lambda: lm.SelectiveScan(s(n, 4, 8), s(n, 4, 8), s(n, 8, 2), s(n, 4, 2), s(n, 4, 2), out=s(n, 4, 8)),
             lambda: lm.SelectiveScan(s(1, 4, 8), s(1, 4, 8), s(1, 8, n), s(1, 4, n), s(1, 4, n), out=s(1, 4, 8)),
             lambda: lm.Orthogonalize(s(1, n, 1), s(1, n, 1, dtype=bf)), lambda: lm.Orthogonalize(s(1, 1, n), s(1, 1, n, dtype=bf)),
             lambda: lm.Orthogonalize(s(n, 1, 1), s(n, 1, 1, dtype=bf)), lambda: lm.Orthogonalize(s(1, 2, 2), s(1, 2, 2, dtype=bf), steps=n)]
    for make in calls:
        _refused(lm, lm.api.ERR_TOO_LARGE, make)
    starts = torch.zeros(n + 1, dtype=torch.int32, device="meta")
    for seq in (lambda: lm._sequences(None, starts, 1, 4, starts.device), lambda: lm._sequences(n, None, 1, 0, starts.device)):
        _refused(lm, lm.api.ERR_TOO_LARGE, seq)


def test_a_wait_that_ran_out_is_reported(lm, devices, monkeypatch):  # noqa: F811
    """The status word reaches the caller: of an operator that is asked, and of a population at its next pull, before any leader is
    followed."""
    from contextlib import nullcontext

    from paper_1905_10395_b200 import lm_population
    real, word = torch.empty, [0]
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: real(*a, **k))
    op = lm.Orthogonalize(torch.zeros(1, 16, 8), torch.zeros(1, 16, 8, dtype=torch.bfloat16))
    op._call = lambda *a: 0

    library = lm.api.lib()

    class Library:
        def __getattr__(self, name):
            return getattr(library, name)

        def lsgd_ortho_check_device(self, f):
            assert devices.current == 1                  # the operator's device, whichever is current
            f._obj.value, was = word[0], word[0]
            word[0] = 0
            return lm.api.ERR_DEVICE_FLAG if was else 0

    monkeypatch.setattr(lm.api, "lib", lambda: Library())
    op.check()
    word[0] = 4
    devices.current = 0
    _refused(lm, lm.api.ERR_DEVICE_FLAG, op.check)
    devices.current = 1
    op.check()                                           # read and cleared

    pop, log = lm_population.LmPopulation.__new__(lm_population.LmPopulation), []

    class Leaders:
        def elect(self, loss):
            log.append("elect")

        def step(self):
            log.append("pull")

    class Step:
        def step(self, lr):
            log.append("adamw")

    x = torch.zeros(1, 16, 8)
    pop.forward, pop._backward, pop._in_order = (lambda a, b: None), (lambda: None), nullcontext
    pop.opt, pop.lsgd, pop.lr, pop.lr_ortho, pop.tau, pop.t = Step(), Leaders(), 0.1, 0.1, 2, 0
    pop.ortho, pop.x, pop.copy = [(op, torch.zeros(1, 16, 8), x, x.clone())], x, x.clone()
    pop.step(None, None)
    word[0] = 4
    _refused(lm, lm.api.ERR_DEVICE_FLAG, lambda: pop.step(None, None))
    assert log == ["adamw", "adamw"]
    pop.step(None, None)
    pop.step(None, None)
    assert log[2:] == ["adamw", "adamw", "elect", "pull"]


def test_plans_are_refused_as_the_calls_are(api):  # noqa: F811
    L, out = api.lib(), (C.c_int32 * 7)()
    for back in (0, 1):
        assert L.lsgd_conv_plan(C.byref(_conv(api)), back, out) == 0 and L.lsgd_scan_plan(C.byref(_scan(api)), back, out) == 0
        assert L.lsgd_conv_plan(C.byref(_conv(api)), back, None) == 1 and L.lsgd_scan_plan(C.byref(_scan(api)), back, None) == 1
        assert L.lsgd_conv_plan(C.byref(_conv(api, W=5)), back, out) == 6 and L.lsgd_scan_plan(C.byref(_scan(api, N=65)), back, out) == 6
        assert L.lsgd_conv_plan(None, back, out) == 1 and L.lsgd_scan_plan(None, back, out) == 1
    assert L.lsgd_ortho_plan(C.byref(_ortho(api)), out) == 0 and L.lsgd_ortho_plan(C.byref(_ortho(api)), None) == 1
    assert L.lsgd_ortho_plan(C.byref(_ortho(api, steps=33)), out) == 6 and L.lsgd_ortho_plan(None, out) == 1
