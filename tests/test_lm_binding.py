"""Host tests of the language-model binding and of the AdamW handle with more devices than the machine has: the current device,
the tensors' device and the CUDA runtime are stand-ins.  No GPU."""
import contextlib
import os
import subprocess
import sys

import pytest
import torch

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Devices:
    """Tensors that count as cuda:1's, a current device, and streams by device and number."""

    def __init__(self, monkeypatch, lm):
        self.current = 1
        self.lm = lm

        @contextlib.contextmanager
        def device(d):
            was, self.current = self.current, torch.device(d).index
            yield
            self.current = was

        monkeypatch.setattr(lm, "_same_device", lambda *t: torch.device("cuda:1"))
        monkeypatch.setattr(lm, "_current_device", lambda: self.current, raising=False)
        monkeypatch.setattr(lm, "_current_stream", lambda index: 0, raising=False)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
        monkeypatch.setattr(torch.cuda, "device", device)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.current)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(torch.device(d), 0))
        monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())


class Stream:
    def __init__(self, device, number):
        self.device, self.cuda_stream = device, number


@pytest.fixture
def lm():
    entry.build()
    from paper_1905_10395_b200 import lm as module
    return module


@pytest.fixture
def devices(monkeypatch, lm):
    return Devices(monkeypatch, lm)


def _operators(lm):
    x = torch.zeros(1, 4, 8)
    yield lm.Embedding(torch.zeros(1, 4, dtype=torch.int64), table=x, out=x, d_out=x, d_table=x)
    yield lm.BlockNorm(x=x, out=x, w_pre=torch.ones(1, 8), h=x, d_h=x, dx=x, rstd_pre=torch.ones(1, 4), stream=Stream(torch.device("cuda:1"), 7))


def test_another_device_is_current(lm, devices, monkeypatch):
    """Nothing reaches the library while another device is current: its default stream has the same handle, 0."""
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: real(*a, **k))
    for op in _operators(lm):
        calls = []
        op._forward = op._backward = lambda *a: calls.append(a) or 0
        devices.current = 0
        for call in (op.forward, op.backward):
            with pytest.raises(lm.api.LsgdError) as e:
                call()
            assert e.value.status == lm.api.ERR_STATE
        assert not calls
        devices.current = 1
        op.forward()
        op.backward()
        assert len(calls) == 2


def test_a_stream_of_another_device(lm, devices):
    x = torch.zeros(1, 4, 8)
    with pytest.raises(lm.api.LsgdError) as e:
        lm.Embedding(torch.zeros(1, 4, dtype=torch.int64), table=x, out=x, stream=Stream(torch.device("cuda:0"), 3))
    assert e.value.status == lm.api.ERR_INVALID_ARG


def test_a_restored_adamw_sets_its_counter_on_its_own_device(lm, devices, monkeypatch):
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: seen.append((name, devices.current)) or 0

    x, state = torch.zeros(256), {k: torch.zeros(256) for k in ("m", "v")}
    monkeypatch.setattr(lm.api, "adamw_state_values", lambda sizes: 256)
    monkeypatch.setattr(lm.api, "lib", lambda: Library())
    devices.current = 0
    opt = lm.AdamW([x], [x], step=5, **state)
    assert seen == [("lsgd_adamw_create", 1), ("lsgd_adamw_set_step", 1)] and devices.current == 0
    opt.h = None


# a CUDA runtime of two devices whose memory is the host's
RUNTIME = r"""
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
static int current = 0;
int fake_synced = -1, fake_freed = -1;
int cudaGetDevice(int* d) { *d = current; return 0; }
int cudaSetDevice(int d) { current = d; return 0; }
int cudaMalloc(void** p, size_t n) { *p = malloc(n); return 0; }
int cudaFree(void* p) { fake_freed = current; free(p); return 0; }
int cudaMemcpyAsync(void* d, const void* s, size_t n, int kind, void* st) { memcpy(d, s, n); return 0; }
int cudaMemcpy(void* d, const void* s, size_t n, int kind) { memcpy(d, s, n); return 0; }
int cudaStreamSynchronize(void* st) { fake_synced = current; return 0; }
"""
PROGRAM = r"""
import ctypes as C, sys
rt, root = C.CDLL(sys.argv[1]), sys.argv[2]
sys.path.insert(0, root)
import numpy as np
from paper_1905_10395_b200 import api
L = api.lib()
size, ptr, wd = np.array([10], dtype=np.int64), np.array([8192], dtype=np.uint64), np.zeros(1, dtype=np.float32)
d = api.AdamwDesc()
d.struct_size, d.n_tensors = C.sizeof(d), 1
d.sizes, d.params, d.grads, d.weight_decay = (a.ctypes.data for a in (size, ptr, ptr, wd))
d.m, d.v, d.beta1, d.beta2, d.eps = 8192, 8192, 0.9, 0.99, 1e-8
h, n = C.c_void_p(), C.c_int64(-1)
rt.cudaSetDevice(1)
assert L.lsgd_adamw_create(C.byref(d), C.byref(h)) == 0
assert L.lsgd_adamw_get_step(h, C.byref(n)) == 0 and n.value == 0
rt.cudaSetDevice(0)
for status in (L.lsgd_adamw_get_step(h, C.byref(n)), L.lsgd_adamw_set_step(h, 3), L.lsgd_adamw_step(h, 0.1, None),
               L.lsgd_adamw_moments(h, None, None)):
    assert status == api.ERR_STATE, status
assert L.lsgd_adamw_destroy(h) == 0
was = C.c_int(-1)
rt.cudaGetDevice(C.byref(was))
assert was.value == 0
assert C.c_int.in_dll(rt, "fake_synced").value == 1 and C.c_int.in_dll(rt, "fake_freed").value == 1
print("done")
"""


def test_an_adamw_handle_belongs_to_its_device(lm, tmp_path):
    """Every call but destroy is refused under another device; destroy waits for and frees on the handle's own."""
    src, so = tmp_path / "rt.c", tmp_path / "librt_two.so"
    src.write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    r = subprocess.run([sys.executable, "-c", PROGRAM, str(so), ROOT], env={**os.environ, "LD_PRELOAD": str(so)}, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr[-2000:]


def test_the_least_eps_of_8_bit_moments(lm):
    """sqrt of the largest second moment that is stored as zero is 2^-50: eps is not below it.  fp32 moments take any normal eps."""
    import ctypes as C

    import numpy as np
    api = lm.api
    size, ptr, wd = np.array([10], dtype=np.int64), np.array([8192], dtype=np.uint64), np.zeros(1, dtype=np.float32)
    for state, eps, refused in ((1, 2.0 ** -51, True), (1, 1e-30, True), (1, 2.0 ** -50, False), (1, 1e-8, False), (0, 2.0 ** -51, False),
                                (0, 1e-30, False), (0, 1e-39, True)):
        d = api.AdamwDesc()
        d.struct_size, d.n_tensors = C.sizeof(d), 1
        d.sizes, d.params, d.grads, d.weight_decay = (a.ctypes.data for a in (size, ptr, ptr, wd))
        d.state_dtype, d.m, d.v, d.m_scale, d.v_scale, d.beta1, d.beta2, d.eps = state, 8192, 8192, 8192, 8192, 0.9, 0.99, eps
        h = C.c_void_p()
        status = api.lib().lsgd_adamw_create(C.byref(d), C.byref(h))
        assert (status == api.ERR_INVALID_ARG) == refused, (state, eps, status)
        if status == 0:
            api.lib().lsgd_adamw_destroy(h)


def test_results_without_their_operand_are_refused(lm, devices):
    """A gradient, or h, whose operand is absent would stay unwritten: the library and the binding refuse it."""
    from tests.test_lm_boundary import _norm
    api = lm.api
    none = api.Rows(None, 0, 0)
    fwd, bwd = api.lib().lsgd_blocknorm_forward, api.lib().lsgd_blocknorm_backward
    import ctypes as C
    assert fwd(C.byref(_norm(api, w_pre=none)), None) == api.ERR_INVALID_ARG                         # h
    for over in (dict(w_pre=none, d_h=none), dict(w_pre=none, d_w_pre=none), dict(post_norm=0), dict(gate_kind=0),
                 dict(y=none, post_norm=0, gate_kind=0, d_w_post=none, d_gate=none)):
        scratch = dict(scratch=8192, scratch_bytes=1 << 40)
        assert bwd(C.byref(_norm(api, **scratch, **over)), None) == api.ERR_INVALID_ARG, over
    t, w = torch.zeros(1, 4, 8), torch.ones(1, 8)
    for kw in (dict(y=t, out=t, h=t, w_post=w), dict(y=t, out=t, d_h=t, w_post=w), dict(y=t, out=t, w_post=w, dw_pre=w),
               dict(y=t, out=t, post_norm=False, dw_post=w), dict(h=t, w_pre=w, dw_post=w), dict(y=t, out=t, w_post=w, d_gate=t),
               dict(h=t, w_pre=w, dy=t)):
        with pytest.raises(api.LsgdError) as e:
            lm.BlockNorm(x=t, **kw)
        assert e.value.status == api.ERR_INVALID_ARG, kw


def test_a_state_is_given_whole(lm, devices, monkeypatch):
    """Codes without their scales would read as zeros, and one moment without the other is no state."""
    class Library:
        def __getattr__(self, name):
            return lambda *a: b"" if name == "lsgd_status_string" else 0

    x, f = torch.zeros(256), torch.zeros(256)
    b, s = torch.zeros(256, dtype=torch.uint8), torch.zeros(1)
    monkeypatch.setattr(lm.api, "adamw_state_values", lambda sizes: 256)
    monkeypatch.setattr(lm.api, "lib", lambda: Library())
    for kw in (dict(m=f), dict(v=f), dict(m=b, v=b), dict(m=b, v=b, m_scale=s), dict(m=b, m_scale=s, state="8bit"),
               dict(v=b, v_scale=s, state="8bit"), dict(m_scale=s, v_scale=s, state="8bit"), dict(m=f, v=f, m_scale=s, v_scale=s)):
        with pytest.raises(lm.api.LsgdError) as e:
            lm.AdamW([x], [x], **kw)
        assert e.value.status == lm.api.ERR_INVALID_ARG, kw
    for kw in (dict(m=f, v=f), dict(m=b, v=b, m_scale=s, v_scale=s)):
        opt = lm.AdamW([x], [x], **kw)
        assert opt.m is kw["m"] and opt.v is kw["v"]
        opt.h = None


def test_tables_of_one_dimension(lm, devices):
    tok, row = torch.zeros(4, dtype=torch.int64), torch.zeros(8)
    for kw in (dict(table=row, out=torch.zeros(4, 8)), dict(d_table=row, d_out=torch.zeros(4, 8))):
        with pytest.raises(lm.api.LsgdError) as e:
            lm.Embedding(tok, **kw)
        assert e.value.status == lm.api.ERR_INVALID_ARG
