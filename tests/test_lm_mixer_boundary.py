"""Host-only checks of the convolution, the scan and the orthogonalisation: struct layouts, refusals before anything is launched,
scratch sizes, the binding's refusals, and the 64-bit restatements against automatic differentiation.  No GPU."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import __graft_entry__ as entry
from tests import _lm_mixer_reference as ref
from tests.test_lm_binding import Devices, Stream

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def api():
    entry.build()
    from paper_1905_10395_b200 import api as a
    return a


@pytest.fixture
def lm(api):
    from paper_1905_10395_b200 import lm as module
    return module


@pytest.fixture
def devices(monkeypatch, lm):
    return Devices(monkeypatch, lm)


def test_struct_layout_matches_header(api, tmp_path):
    kinds = {"lsgd_sequences": api.Sequences, "lsgd_conv_desc": api.ConvDesc, "lsgd_scan_desc": api.ScanDesc, "lsgd_ortho_desc": api.OrthoDesc}
    fields = [("lsgd_sequences", "S"), ("lsgd_conv_desc", "seq"), ("lsgd_conv_desc", "state"), ("lsgd_conv_desc", "scratch_bytes"),
              ("lsgd_scan_desc", "x"), ("lsgd_scan_desc", "a_log"), ("lsgd_scan_desc", "saved"), ("lsgd_scan_desc", "d_dt_bias"),
              ("lsgd_scan_desc", "scratch_bytes"), ("lsgd_ortho_desc", "scale"), ("lsgd_ortho_desc", "grad"), ("lsgd_ortho_desc", "scratch_bytes")]
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "lsgd.h"\nint main(void){'
                   + "".join(f'printf("%zu ",sizeof({n}));' for n in kinds)
                   + "".join(f'printf("%zu ",offsetof({n},{f}));' for n, f in fields) + "return 0;}\n")
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(k) for k in kinds.values()] + [getattr(kinds[n], f).offset for n, f in fields]


MB = 1 << 20


def _conv(api, **over):
    d = api.ConvDesc()
    d.struct_size = C.sizeof(d)
    d.P, d.T, d.D, d.W, d.act_dtype, d.act = 2, 100, 16, 4, 1, 1
    d.seq = api.Sequences(None, 0, 5)
    for i, k in enumerate(("x", "out", "d_out", "dx")):
        setattr(d, k, api.Rows((i + 1) * MB, 16, 1600))
    d.w, d.dw = api.Rows(5 * MB, 4, 64), api.Rows(6 * MB, 4, 64)
    d.bias, d.d_bias = api.Rows(7 * MB, 0, 16), api.Rows(8 * MB, 0, 16)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def _scan(api, **over):
    d = api.ScanDesc()
    d.struct_size = C.sizeof(d)
    d.P, d.T, d.D, d.N, d.act_dtype = 2, 100, 16, 8, 1
    d.seq = api.Sequences(None, 0, 5)
    at = iter(range(1, 100))
    for k in ("x", "dt", "z", "out", "d_out", "dx", "d_dt", "dz"):
        setattr(d, k, api.Rows(next(at) * MB, 16, 1600))
    for k in ("b", "c", "db", "dc"):
        setattr(d, k, api.Rows(next(at) * MB, 8, 800))
    d.a_log, d.d_a_log = api.Rows(next(at) * MB, 8, 128), api.Rows(next(at) * MB, 8, 128)
    for k in ("skip", "dt_bias", "d_skip", "d_dt_bias"):
        setattr(d, k, api.Rows(next(at) * MB, 0, 16))
    d.saved = next(at) * MB
    for k, v in over.items():
        setattr(d, k, v)
    return d


def _ortho(api, **over):
    d = api.OrthoDesc()
    d.struct_size = C.sizeof(d)
    d.P, d.m, d.n, d.steps, d.nesterov = 2, 30, 200, 5, 1
    d.a, d.b, d.c, d.mu, d.eps, d.scale = 3.4445, -4.775, 2.0315, 0.95, 1e-7, 1.0
    d.grad, d.momentum, d.out = api.Rows(MB, 200, 6000), api.Rows(2 * MB, 200, 6000), api.Rows(3 * MB, 200, 6000)
    for k, v in over.items():
        setattr(d, k, v)
    return d


nan, inf = float("nan"), float("inf")
COMMON = [(dict(struct_size=8), 1), (dict(P=0), 1), (dict(T=-1), 1), (dict(D=0), 1), (dict(act_dtype=2), 1), (dict(act_dtype=-1), 1),
          (dict(D=65537), 6), (dict(P=65536), 6), (dict(T=1 << 30), 8), (dict(T=101), 1)]
CONV_BAD = COMMON + [(dict(W=0), 1), (dict(W=5), 6), (dict(act=2), 1), (dict(act=-1), 1)]
SCAN_BAD = COMMON + [(dict(N=0), 1), (dict(N=65), 6), (dict(saved=MB + 8), 3)]
ORTHO_BAD = [(dict(struct_size=8), 1), (dict(P=0), 1), (dict(m=0), 1), (dict(n=0), 1), (dict(steps=-1), 1), (dict(steps=33), 6), (dict(P=65536), 6),
             (dict(m=65537), 6), (dict(m=65536, n=65536), 8), (dict(grad_dtype=2), 1), (dict(a=17.0), 1), (dict(b=nan), 1), (dict(c=-inf), 1),
             (dict(mu=1.0), 1), (dict(mu=-0.1), 1), (dict(mu=nan), 1), (dict(eps=-1.0), 1), (dict(eps=nan), 1), (dict(scale=inf), 1)]


@pytest.mark.parametrize("over,status", CONV_BAD)
def test_conv_refuses(api, over, status):
    for f in (api.lib().lsgd_conv_forward, api.lib().lsgd_conv_backward):
        assert f(C.byref(_conv(api, **over)), None) == status


@pytest.mark.parametrize("over,status", SCAN_BAD)
def test_scan_refuses(api, over, status):
    for f in (api.lib().lsgd_scan_forward, api.lib().lsgd_scan_backward):
        assert f(C.byref(_scan(api, **over)), None) == status


@pytest.mark.parametrize("over,status", ORTHO_BAD)
def test_ortho_refuses(api, over, status):
    assert api.lib().lsgd_ortho(C.byref(_ortho(api, **over)), None) == status


def test_sequences_are_checked(api):
    S = api.Sequences
    for make, calls in ((_conv, (api.lib().lsgd_conv_forward, api.lib().lsgd_conv_backward)),
                        (_scan, (api.lib().lsgd_scan_forward, api.lib().lsgd_scan_backward))):
        for seq, status in ((S(None, 0, 0), 1), (S(None, 0, -2), 1), (S(None, 0, 3), 1), (S(8194, 6, 5), 3), (S(8192, -1, 5), 1), (S(8192, 5, 5), 1),
                            (S(8192, 1 << 60, 5), 8)):
            for call in calls:
                assert call(C.byref(make(api, seq=seq)), None) == status, (make, seq.starts, seq.stride, seq.S)


def test_most_rows(api):
    """2^31 - 2^20 rows are too many; one less passes, to the refusal of the scratch's alignment."""
    L, T = api.lib(), (1 << 31) - (1 << 20)
    rows = dict(P=1, seq=api.Sequences(1 << 50, 0, 5), scratch=8, scratch_bytes=1 << 60)
    far = {k: api.Rows((1 + i) << 42, 16, 0) for i, k in enumerate(("x", "dt", "z", "out", "d_out", "dx", "d_dt", "dz", "b", "c", "db", "dc"))}
    for make, calls in ((_conv, (L.lsgd_conv_forward, L.lsgd_conv_backward)), (_scan, (L.lsgd_scan_forward, L.lsgd_scan_backward))):
        names = {f for f, _ in type(make(api))._fields_}
        over = rows | {k: v for k, v in far.items() if k in names} | ({"saved": 1 << 52} if "saved" in names else {})
        for call in calls:
            assert call(C.byref(make(api, T=T, **over)), None) == 8 and call(C.byref(make(api, T=T - 1, **over)), None) == 3


def test_conv_refuses_rows(api):
    fwd, bwd = api.lib().lsgd_conv_forward, api.lib().lsgd_conv_backward
    R = api.Rows
    none = R(None, 0, 0)
    for k in ("x", "w", "out"):
        assert fwd(C.byref(_conv(api, **{k: none})), None) == 1, k
    for k in ("x", "w", "d_out", "dx", "dw", "d_bias", "bias"):          # a bias and its gradient are given together
        assert bwd(C.byref(_conv(api, **{k: none})), None) == 1, k
    for r, status in ((R(MB + 1, 16, 1600), 3), (R(MB, -16, 1600), 1), (R(MB, 1 << 60, 1600), 8)):
        assert fwd(C.byref(_conv(api, x=r)), None) == status
    for r, status in ((R(2 * MB, 15, 1600), 1), (R(2 * MB, 16, 0), 1), (R(2 * MB, 0, 1600), 1)):
        assert fwd(C.byref(_conv(api, out=r)), None) == status
    assert fwd(C.byref(_conv(api, state=MB * 20 + 1)), None) == 3
    assert bwd(C.byref(_conv(api, state=MB * 20)), None) == 1            # no gradient through a state
    assert bwd(C.byref(_conv(api, dw=R(6 * MB, 3, 64))), None) == 1
    need = api.lib().lsgd_conv_scratch_bytes(C.byref(_conv(api)), 1)
    assert need > 0 and api.lib().lsgd_conv_scratch_bytes(C.byref(_conv(api)), 0) == 0
    assert bwd(C.byref(_conv(api)), None) == 1
    assert bwd(C.byref(_conv(api, scratch=MB * 30, scratch_bytes=need - 1)), None) == 1
    assert bwd(C.byref(_conv(api, scratch=MB * 30 + 128, scratch_bytes=need)), None) == 3
    ragged = dict(seq=api.Sequences(MB * 31, 0, 5))
    assert api.lib().lsgd_conv_scratch_bytes(C.byref(_conv(api, **ragged)), 0) >= 4 * 200
    assert fwd(C.byref(_conv(api, **ragged)), None) == 1                 # the table of rows needs scratch
    assert fwd(None, None) == 1 and bwd(None, None) == 1 and api.lib().lsgd_conv_scratch_bytes(None, 0) == 0


def test_scan_refuses_rows(api):
    fwd, bwd = api.lib().lsgd_scan_forward, api.lib().lsgd_scan_backward
    R = api.Rows
    none = R(None, 0, 0)
    for k in ("x", "dt", "b", "c", "a_log", "out"):
        assert fwd(C.byref(_scan(api, **{k: none})), None) == 1, k
    for k in ("x", "dt", "b", "c", "a_log", "d_out", "dx", "d_dt", "db", "dc", "d_a_log", "z", "dz", "skip", "d_skip", "dt_bias", "d_dt_bias"):
        assert bwd(C.byref(_scan(api, **{k: none})), None) == 1, k
    assert bwd(C.byref(_scan(api, saved=None)), None) == 1 and bwd(C.byref(_scan(api, state=MB * 50)), None) == 1
    assert fwd(C.byref(_scan(api, state=MB * 50 + 4)), None) == 3
    need = api.lib().lsgd_scan_scratch_bytes(C.byref(_scan(api)), 1)
    assert bwd(C.byref(_scan(api, scratch=MB * 60, scratch_bytes=need - 1)), None) == 1
    assert bwd(C.byref(_scan(api, scratch=MB * 60 + 8, scratch_bytes=need)), None) == 3
    assert fwd(None, None) == 1 and bwd(None, None) == 1 and api.lib().lsgd_scan_scratch_bytes(None, 0) == 0


def test_outputs_overlap_no_input(api):
    """Columns of one buffer are apart, shifted rows of it are not."""
    R = api.Rows
    conv, scan = api.lib().lsgd_conv_forward, api.lib().lsgd_scan_forward
    assert conv(C.byref(_conv(api, out=R(MB, 16, 1600))), None) == 1                                  # in place
    assert conv(C.byref(_conv(api, out=R(MB + 32, 16, 1600))), None) == 1                             # a row on
    assert conv(C.byref(_conv(api, x=R(MB, 32, 3200), out=R(MB + 16, 32, 3200))), None) == 1          # half a row on
    assert conv(C.byref(_conv(api, x=R(MB, 32, 3200), out=R(MB + 32, 64, 6400))), None) == 1          # other strides: not certain
    assert conv(C.byref(_conv(api, state=2 * MB)), None) == 1
    assert scan(C.byref(_scan(api, out=R(2 * MB, 16, 1600))), None) == 1 and scan(C.byref(_scan(api, state=MB)), None) == 1
    bwd = api.lib().lsgd_scan_backward
    assert bwd(C.byref(_scan(api, dx=R(5 * MB, 16, 1600))), None) == 1                                # the incoming gradient's place
    assert bwd(C.byref(_scan(api, dx=R(7 * MB, 16, 1600))), None) == 1                                # another result's
    # columns of one buffer pass: the next refusal is the missing scratch
    ragged = dict(seq=api.Sequences(MB * 70, 0, 5))
    assert conv(C.byref(_conv(api, x=R(MB, 32, 3200), out=R(MB + 32, 32, 3200), scratch=MB * 30 + 8, scratch_bytes=1 << 30, **ragged)), None) == 3
    assert conv(C.byref(_conv(api, x=R(MB, 64, 32), out=R(MB + 32, 64, 32), scratch=MB * 30 + 8, scratch_bytes=1 << 30, **ragged)), None) == 3
    # parameters, and the saved states that the backward pass reads, are inputs too
    assert conv(C.byref(_conv(api, out=R(5 * MB, 16, 1600))), None) == 1 and conv(C.byref(_conv(api, out=R(7 * MB, 16, 1600))), None) == 1
    d = _scan(api)
    for at in (d.a_log.data, d.skip.data, d.dt_bias.data):
        assert scan(C.byref(_scan(api, out=R(at, 16, 1600))), None) == 1
    assert bwd(C.byref(_scan(api, d_dt=R(d.saved, 16, 1600))), None) == 1
    ortho = api.lib().lsgd_ortho
    for k, r in (("out", R(MB, 200, 6000)), ("momentum", R(MB, 200, 6000)), ("out", R(2 * MB + 4, 200, 6000))):
        assert ortho(C.byref(_ortho(api, **{k: r})), None) == 1


def test_ortho_refuses_rows(api):
    ortho, R = api.lib().lsgd_ortho, api.Rows
    none = R(None, 0, 0)
    assert ortho(C.byref(_ortho(api, grad=none)), None) == 1 and ortho(C.byref(_ortho(api, out=none)), None) == 1
    assert ortho(C.byref(_ortho(api, grad=R(MB + 2, 200, 6000))), None) == 3
    assert ortho(C.byref(_ortho(api, momentum=R(2 * MB, 199, 6000))), None) == 1
    assert ortho(C.byref(_ortho(api, out=R(3 * MB, 200, 0))), None) == 1
    big = dict(m=300, n=400, grad=R(MB, 400, 120000), momentum=none, out=R(3 * MB, 400, 120000))
    need = api.lib().lsgd_ortho_scratch_bytes(C.byref(_ortho(api, **big)))
    assert need > 0 and ortho(C.byref(_ortho(api, **big)), None) == 1
    assert ortho(C.byref(_ortho(api, scratch=MB * 9, scratch_bytes=need - 1, **big)), None) == 1
    assert ortho(C.byref(_ortho(api, scratch=MB * 9 + 16, scratch_bytes=need, **big)), None) == 3
    assert ortho(None, None) == 1 and api.lib().lsgd_ortho_scratch_bytes(None) == 0


# ---- the binding
def _refused(lm, status, make):
    with pytest.raises(lm.api.LsgdError) as e:
        make()
    assert e.value.status == status


def test_binding_refuses(lm, devices):
    bad, unsupported = lm.api.ERR_INVALID_ARG, lm.api.ERR_UNSUPPORTED
    x, w, o = torch.zeros(2, 12, 8), torch.zeros(2, 8, 4), torch.zeros(2, 12, 8)
    conv = lambda *a, **k: (lambda: lm.CausalConv(*a, **k))  # noqa: E731
    starts = torch.tensor([0, 5, 12], dtype=torch.int32)
    monkey = starts.to("meta")
    for make in (conv(x, w), conv(x, w, out=o, act="relu"), conv(x, w, out=o, sequences=5), conv(x, w, out=o, sequences=0),
                 conv(x, w, out=torch.zeros(2, 11, 8)), conv(x, w, out=o, sequences=2, starts=starts), conv(x, w, out=o, d_out=x),
                 conv(x, w, out=o, state=torch.zeros(2, 1, 2, 8)), conv(x, torch.zeros(2, 7, 4), out=o), conv(x, w, out=o, starts=monkey),
                 conv(x, w, d_out=o, dx=o, dw=w, state=torch.zeros(2, 1, 3, 8)), conv(x, w, d_out=o, dx=o, dw=w, bias=torch.zeros(2, 8)),
                 conv(x[0, 0], w, out=o), conv(x.transpose(1, 2), w.transpose(1, 2), out=o)):
        _refused(lm, bad, make)
    for make in (conv(x.half(), w, out=o.half()), conv(x, w.double(), out=o), conv(x, w, out=o, state=torch.zeros(2, 1, 3, 8).bfloat16()),
                 conv(x, w, out=o, starts=starts.long())):
        if make is not None:
            with pytest.raises(lm.api.LsgdError):
                make()
    a, bc = torch.zeros(2, 8, 4), torch.zeros(2, 12, 4)
    scan = lambda *p, **k: (lambda: lm.SelectiveScan(*p, **k))  # noqa: E731
    grads = dict(d_out=o, d_x=o, d_dt=o, d_a_log=a, d_b=bc, d_c=bc)
    for make in (scan(x, x, a, bc, bc), scan(x, x, a, bc, torch.zeros(2, 12, 5), out=o), scan(x, x, a, bc, bc, out=o, d_out=o),
                 scan(x, x, a, bc, bc, z=x, **grads), scan(x, x, a, bc, bc, skip=torch.zeros(2, 8), **grads),
                 scan(x, x, a, bc, bc, d_dt_bias=torch.zeros(2, 8), **grads), scan(x, x, a, bc, bc, state=torch.zeros(2, 1, 8, 4), **grads),
                 scan(x, x, a, bc, bc, out=o, state=torch.zeros(2, 2, 8, 4)), scan(x, x, a, bc, bc, out=o, saved=torch.zeros(2, 1, 8, 4))):
        _refused(lm, bad, make)
    _refused(lm, unsupported, scan(x, x, a.double(), bc, bc, out=o))
    ortho = lambda *p, **k: (lambda: lm.Orthogonalize(*p, **k))  # noqa: E731
    g, out = torch.zeros(2, 6, 9), torch.zeros(2, 6, 9, dtype=torch.bfloat16)
    for make in (ortho(g, out[:, :5]), ortho(g, out, coefficients=(1.0, 2.0)), ortho(g, out, momentum=g[:, :, :8])):
        _refused(lm, bad, make)
    for make in (ortho(g, g), ortho(g.double(), out), ortho(g, out, momentum=g.bfloat16())):
        _refused(lm, unsupported, make)


def test_another_device_is_current(lm, devices, monkeypatch):
    real = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: real(*a, **k))
    x, w, g = torch.zeros(1, 16, 8), torch.zeros(1, 8, 4), torch.zeros(1, 16, 8)
    bc, out = torch.zeros(1, 16, 4), torch.zeros(1, 16, 8, dtype=torch.bfloat16)
    ops = [lm.CausalConv(x, w, out=g, stream=Stream(torch.device("cuda:1"), 7)), lm.SelectiveScan(x, x, w, bc, bc, out=g), lm.Orthogonalize(x, out)]
    for op in ops:
        calls = []
        op._forward = op._call = lambda *a: calls.append(a) or 0
        devices.current = 0
        with pytest.raises(lm.api.LsgdError) as e:
            op.forward()
        assert e.value.status == lm.api.ERR_STATE and not calls
        devices.current = 1
        op.forward()
        assert len(calls) == 1


# ---- the 64-bit restatements
def _leaf(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64).requires_grad_()


def test_reference_scan_against_automatic_differentiation():
    gen = torch.Generator().manual_seed(0)
    P, T, D, N = 2, 12, 3, 4
    t = {k: _leaf(gen, P, T, D) for k in ("x", "dt", "z")} | {k: _leaf(gen, P, T, N) for k in ("b", "c")}
    t |= {"a_log": _leaf(gen, P, D, N), "skip": _leaf(gen, P, D), "dt_bias": _leaf(gen, P, D)}
    up = torch.randn((P, T, D), generator=gen, dtype=torch.float64)
    edges = [[0, 5, 5, 12], [2, 3, 11, 11]]
    outs = torch.zeros((P, T, D), dtype=torch.float64)
    for p in range(P):
        for lo, hi in zip(edges[p], edges[p][1:]):
            h = torch.zeros((D, N), dtype=torch.float64)
            for i in range(lo, hi):
                delta = torch.nn.functional.softplus(t["dt"][p, i] + t["dt_bias"][p])
                h = torch.exp(-delta[:, None] * torch.exp(t["a_log"][p])) * h + (delta * t["x"][p, i])[:, None] * t["b"][p, i]
                y = (h * t["c"][p, i]).sum(-1) + t["skip"][p] * t["x"][p, i]
                outs = outs.index_put((torch.tensor(p), torch.tensor(i)), y * torch.nn.functional.silu(t["z"][p, i]))
    (outs * up).sum().backward()
    d = {k: v.detach() for k, v in t.items()}
    got, size = ref.scan(d["x"], d["dt"], d["a_log"], d["b"], d["c"], d["z"], d["skip"], d["dt_bias"], None, up, edges)
    live = ~torch.isnan(got["out"])
    assert live.sum() == (12 + 9) * D and (got["out"][live] - outs[live]).abs().max() < 1e-13
    for k, v in t.items():
        g = torch.nan_to_num(got["d_" + k])
        assert (g - v.grad).abs().max() < 1e-12, k
        assert (torch.nan_to_num(size["d_" + k]) >= g.abs() - 1e-12).all()


@pytest.mark.parametrize("act", ["silu", "identity"])
def test_reference_conv_against_automatic_differentiation(act):
    gen = torch.Generator().manual_seed(1)
    P, T, D, W = 2, 11, 3, 4
    x, w, bias = _leaf(gen, P, T, D), _leaf(gen, P, D, W), _leaf(gen, P, D)
    up = torch.randn((P, T, D), generator=gen, dtype=torch.float64)
    edges = [[0, 2, 2, 11], [1, 7, 8, 8]]
    total = 0.0
    for p in range(P):
        for lo, hi in zip(edges[p], edges[p][1:]):
            if hi > lo:
                pre = torch.nn.functional.conv1d(x[p, lo:hi].T[None], w[p][:, None], bias[p], padding=W - 1, groups=D)[0, :, :hi - lo].T
                total = total + ((torch.nn.functional.silu(pre) if act == "silu" else pre) * up[p, lo:hi]).sum()
    total.backward()
    got, _ = ref.conv(x.detach(), w.detach(), bias.detach(), None, up, edges, act)
    assert abs(torch.nansum(got["out"] * up).item() - total.item()) < 1e-11
    for k, v in (("dx", x), ("dw", w), ("d_bias", bias)):
        assert (torch.nan_to_num(got[k]) - v.grad).abs().max() < 1e-12, k


def test_reference_ortho_maps_singular_values():
    gen = torch.Generator().manual_seed(2)
    for m, n in ((5, 9), (9, 5)):
        g = torch.randn((2, m, n), generator=gen, dtype=torch.float64)
        out, _ = ref.ortho(g, steps=3, eps=0.0)
        u, s, vh = torch.linalg.svd(g / torch.linalg.matrix_norm(g)[:, None, None], full_matrices=False)
        for _ in range(3):
            s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
        assert ((u * s[:, None]) @ vh - out).abs().max() < 1e-12
