"""Host-only checks of the language-model operators: struct layouts, refusals before anything is launched, sizes.  No GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from tests import _lm_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def api():
    entry.build()
    from paper_1905_10395_b200 import api as a
    return a


def test_struct_layout_matches_header(api, tmp_path):
    names = ["lsgd_rows", "lsgd_embed_desc", "lsgd_blocknorm_desc", "lsgd_adamw_desc"]
    ends = [("lsgd_embed_desc", "scratch_bytes"), ("lsgd_embed_desc", "table"), ("lsgd_blocknorm_desc", "scratch_bytes"),
            ("lsgd_blocknorm_desc", "rstd_post"), ("lsgd_blocknorm_desc", "x"), ("lsgd_adamw_desc", "stream"), ("lsgd_adamw_desc", "beta1")]
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "lsgd.h"\nint main(void){'
                   + "".join(f'printf("%zu ",sizeof({n}));' for n in names)
                   + "".join(f'printf("%zu ",offsetof({n},{f}));' for n, f in ends) + "return 0;}\n")
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    kinds = {"lsgd_rows": api.Rows, "lsgd_embed_desc": api.EmbedDesc, "lsgd_blocknorm_desc": api.BlocknormDesc, "lsgd_adamw_desc": api.AdamwDesc}
    assert got == [C.sizeof(kinds[n]) for n in names] + [getattr(kinds[n], f).offset for n, f in ends]


# ---- embedding
def _embed(api, **over):
    e = api.EmbedDesc()
    e.struct_size = C.sizeof(e)
    e.P, e.T, e.V, e.D, e.token_bytes, e.padding, e.scale = 2, 100, 50, 16, 8, -1, 1.0
    e.tokens, e.token_stride = 4096, 100
    e.table, e.out = api.Rows(8192, 16, 800), api.Rows(8192, 16, 1600)
    e.d_out, e.d_table = api.Rows(8192, 16, 1600), api.Rows(8192, 16, 800)
    for k, v in over.items():
        setattr(e, k, v)
    return e


EMBED_BAD = [(dict(struct_size=8), 1), (dict(P=0), 1), (dict(T=-1), 1), (dict(V=0), 1), (dict(D=0), 1), (dict(token_bytes=2), 1),
             (dict(table_dtype=2), 1), (dict(act_dtype=-1), 1), (dict(padding=-2), 1), (dict(padding=50), 1), (dict(tokens=None), 1),
             (dict(token_stride=-1), 1), (dict(tokens=4100), 3), (dict(D=65537), 6), (dict(T=1 << 30), 8), (dict(V=1 << 30), 8)]


@pytest.mark.parametrize("over,status", EMBED_BAD)
def test_embed_refuses(api, over, status):
    for f in (api.lib().lsgd_embed_forward, api.lib().lsgd_embed_backward):
        assert f(C.byref(_embed(api, **over)), None) == status


def test_embed_refuses_rows(api):
    fwd, bwd = api.lib().lsgd_embed_forward, api.lib().lsgd_embed_backward
    R = api.Rows
    for rows, status in ((R(None, 16, 1600), 1), (R(8194, 16, 1600), 3), (R(8192, -16, 1600), 1), (R(8192, 16, -1), 1),
                         (R(8192, 15, 1600), 1), (R(8192, 16, 1599), 1), (R(8192, 0, 1600), 1), (R(8192, 16, 0), 1),
                         (R(8192, 1 << 60, 1600), 8)):
        assert fwd(C.byref(_embed(api, out=rows)), None) == status
    for rows, status in ((R(None, 16, 800), 1), (R(8194, 16, 800), 3), (R(8192, 15, 800), 1), (R(8192, 16, 799), 1)):
        assert bwd(C.byref(_embed(api, d_table=rows)), None) == status
    assert bwd(C.byref(_embed(api, T=5000, token_stride=5000, d_out=R(8192, 16, 80000))), None) == 1      # no scratch
    need = api.lib().lsgd_embed_scratch_bytes(C.byref(_embed(api, T=5000)))
    assert need > 0 and api.lib().lsgd_embed_scratch_bytes(C.byref(_embed(api))) == 0
    big = dict(T=5000, token_stride=5000, d_out=R(8192, 16, 80000))
    assert bwd(C.byref(_embed(api, scratch=8192, scratch_bytes=need - 1, **big)), None) == 1
    assert bwd(C.byref(_embed(api, scratch=8192 + 128, scratch_bytes=need, **big)), None) == 3
    assert fwd(None, None) == 1 and bwd(None, None) == 1
    assert api.lib().lsgd_embed_scratch_bytes(None) == 0 and api.lib().lsgd_embed_scratch_bytes(C.byref(_embed(api, P=0))) == 0


# ---- block-boundary norms
def _norm(api, **over):
    d = api.BlocknormDesc()
    d.struct_size = C.sizeof(d)
    d.P, d.T, d.D, d.resid_dtype, d.act_dtype = 2, 10, 64, 0, 1
    d.post_norm, d.gate_kind, d.alpha, d.beta, d.eps = 1, 2, 1.0, 1.0, 1e-6
    f, v = api.Rows(8192, 64, 640), api.Rows(8192, 0, 64)
    for k in ("x", "y", "gate", "out", "h", "d_out", "d_h", "dx", "dy", "d_gate"):
        setattr(d, k, f)
    for k in ("w_post", "w_pre", "d_w_post", "d_w_pre"):
        setattr(d, k, v)
    d.rstd_post = d.rstd_pre = 8192
    for k, x in over.items():
        setattr(d, k, x)
    return d


NORM_BAD = [(dict(struct_size=4), 1), (dict(P=0), 1), (dict(T=-1), 1), (dict(D=0), 1), (dict(resid_dtype=3), 1), (dict(act_dtype=-1), 1),
            (dict(resid_dtype=1, act_dtype=0), 6), (dict(D=8193), 6), (dict(P=70000), 6), (dict(T=1 << 30), 8), (dict(gate_kind=3), 1),
            (dict(gate_act=3), 1), (dict(eps=0.0), 1), (dict(eps=float("nan")), 1), (dict(eps=-1.0), 1), (dict(alpha=float("inf")), 1),
            (dict(beta=float("nan")), 1), (dict(rstd_post=None), 1), (dict(rstd_pre=None), 1), (dict(rstd_pre=8193), 3)]


@pytest.mark.parametrize("over,status", NORM_BAD)
def test_blocknorm_refuses(api, over, status):
    for f in (api.lib().lsgd_blocknorm_forward, api.lib().lsgd_blocknorm_backward):
        assert f(C.byref(_norm(api, **over)), None) == status


def test_blocknorm_refuses_rows(api):
    fwd, bwd = api.lib().lsgd_blocknorm_forward, api.lib().lsgd_blocknorm_backward
    R = api.Rows
    none = R(None, 0, 0)
    for k in ("x", "out", "h", "gate", "w_post"):
        assert fwd(C.byref(_norm(api, **{k: none})), None) == 1, k
    assert fwd(C.byref(_norm(api, y=none)), None) == 1                            # a gate and a norm of nothing
    assert fwd(C.byref(_norm(api, y=none, post_norm=0, gate_kind=0, w_pre=none)), None) == 1   # nothing to compute
    for k in ("out", "h"):
        assert fwd(C.byref(_norm(api, **{k: R(8192, 63, 640)})), None) == 1
        assert fwd(C.byref(_norm(api, **{k: R(8192, 64, 0)})), None) == 1
        assert fwd(C.byref(_norm(api, **{k: R(8193, 64, 640)})), None) == 3
    for k in ("dx", "dy", "d_h", "out", "d_gate"):
        assert bwd(C.byref(_norm(api, **{k: none})), None) == 1, k
    assert bwd(C.byref(_norm(api, d_w_pre=R(8192, 0, 63))), None) == 1
    assert bwd(C.byref(_norm(api)), None) == 1                                    # no scratch
    need = api.lib().lsgd_blocknorm_scratch_bytes(C.byref(_norm(api)))
    assert need > 0 and bwd(C.byref(_norm(api, scratch=8192, scratch_bytes=need - 1)), None) == 1
    assert bwd(C.byref(_norm(api, scratch=8200, scratch_bytes=need)), None) == 3
    assert fwd(None, None) == 1 and bwd(None, None) == 1 and api.lib().lsgd_blocknorm_scratch_bytes(None) == 0


# ---- AdamW
def _adamw(api, **over):
    sizes = np.array([10, 300], dtype=np.int64)
    ptrs = np.array([8192, 16384], dtype=np.uint64)
    wd = np.zeros(2, dtype=np.float32)
    d = api.AdamwDesc()
    d.struct_size, d.n_tensors = C.sizeof(d), 2
    d.sizes, d.params, d.grads, d.weight_decay = (a.ctypes.data for a in (sizes, ptrs, ptrs, wd))
    d.state_dtype, d.m, d.v, d.m_scale, d.v_scale = 1, 8192, 8192, 8192, 8192
    d.beta1, d.beta2, d.eps = 0.9, 0.99, 1e-8
    keep = [sizes, ptrs, wd]
    for k, v in over.items():
        if isinstance(v, np.ndarray):
            keep.append(v)
            v = v.ctypes.data
        setattr(d, k, v)
    return d, keep


ADAMW_BAD = [(dict(struct_size=8), 1), (dict(n_tensors=0), 1), (dict(sizes=None), 1), (dict(params=None), 1), (dict(grads=None), 1),
             (dict(weight_decay=None), 1), (dict(grad_dtype=2), 1), (dict(state_dtype=2), 1), (dict(beta1=1.0), 1), (dict(beta2=-0.1), 1),
             (dict(beta1=float("nan")), 1), (dict(eps=0.0), 1), (dict(eps=1e-60), 1), (dict(eps=float("inf")), 1), (dict(m=None), 1),
             (dict(v=None), 1), (dict(m_scale=None), 1), (dict(v_scale=None), 1), (dict(m=8192 + 16), 3), (dict(v=8200), 3),
             (dict(m_scale=8193), 3), (dict(sizes=np.array([10, -1], dtype=np.int64)), 1),
             (dict(params=np.array([8192, 0], dtype=np.uint64)), 1), (dict(grads=np.array([0, 8192], dtype=np.uint64)), 1),
             (dict(params=np.array([8192, 8194], dtype=np.uint64)), 3), (dict(copies=np.array([8193, 0], dtype=np.uint64)), 3),
             (dict(weight_decay=np.array([0, np.inf], dtype=np.float32)), 1), (dict(sizes=np.array([1 << 49, 1], dtype=np.int64)), 1)]


@pytest.mark.parametrize("over,status", ADAMW_BAD)
def test_adamw_refuses(api, over, status):
    d, keep = _adamw(api, **over)
    h = C.c_void_p(123)
    assert api.lib().lsgd_adamw_create(C.byref(d), C.byref(h)) == status
    assert h.value is None


def test_adamw_handles_and_sizes(api):
    L = api.lib()
    assert L.lsgd_adamw_create(None, C.byref(C.c_void_p())) == 1 and L.lsgd_adamw_create(C.byref(_adamw(api)[0]), None) == 1
    assert L.lsgd_adamw_step(None, 0.1, None) == 1 and L.lsgd_adamw_moments(None, None, None) == 1
    assert L.lsgd_adamw_get_step(None, None) == 1 and L.lsgd_adamw_set_step(None, 0) == 1 and L.lsgd_adamw_destroy(None) == 0
    assert api.adamw_state_values([1, 256, 257, 0]) == 256 + 256 + 512
    with pytest.raises(api.LsgdError):
        api.adamw_state_values([-1])
    if not torch.cuda.is_available():
        h = C.c_void_p()
        d, keep = _adamw(api)
        assert L.lsgd_adamw_create(C.byref(d), C.byref(h)) == api.ERR_CUDA and h.value is None


# ---- the binding refuses what the library would not see
def test_binding_refuses(api):
    from paper_1905_10395_b200 import lm
    x = torch.zeros(1, 4, 8)
    with pytest.raises(api.LsgdError):                      # no CPU path
        lm.Embedding(torch.zeros(1, 4, dtype=torch.int64), table=x, out=x)
    with pytest.raises(api.LsgdError):
        lm.BlockNorm(x=x, h=x, w_pre=torch.ones(1, 8))
    with pytest.raises(api.LsgdError):
        lm.AdamW([x], [x])
    with pytest.raises(api.LsgdError):
        lm.Embedding(torch.zeros(1, 4, dtype=torch.int16), table=x, out=x)
    with pytest.raises(api.LsgdError):
        lm.AdamW([], [])


# ---- the references that the GPU tests lean on
@pytest.mark.parametrize("gate", [None, "channel", "token"])
@pytest.mark.parametrize("act", ["identity", "sigmoid", "tanh"])
def test_reference_gradients_are_those_of_the_reference_forward(gate, act):
    gen = torch.Generator().manual_seed(1)
    mk = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64, requires_grad=True)  # noqa: E731
    P, T, D = 2, 3, 10
    v = {"x": mk(P, T, D), "y": mk(P, T, D), "w_post": mk(P, D), "w_pre": mk(P, D)}
    if gate:
        v["gate"] = mk(P, D) if gate == "channel" else mk(P, T, D)
    c1, c2 = mk(P, T, D).detach(), mk(P, T, D).detach()
    opt = dict(act=act, alpha=0.7, beta=1.3, eps=1e-2)
    out, h = ref.blocknorm_forward(v["x"], v["y"], v.get("gate"), v["w_post"], v["w_pre"], **opt)
    ((c1 * out).sum() + (c2 * h).sum()).backward()
    d = {k: t.detach() for k, t in v.items() if k != "x"}
    got, _ = ref.blocknorm_backward(c1, c2, out.detach(), **d, **opt)
    for name, k in (("dx", "x"), ("dy", "y"), ("dw_post", "w_post"), ("dw_pre", "w_pre"), ("d_gate", "gate")):
        if k in v:
            assert torch.allclose(got[name], v[k].grad, rtol=1e-10, atol=1e-12), name


def test_reference_embedding_gradient():
    gen = torch.Generator().manual_seed(2)
    table = torch.randn((2, 5, 3), generator=gen, dtype=torch.float64, requires_grad=True)
    tok = torch.tensor([[0, 4, 4, 2], [1, 1, 1, 3]])
    c = torch.randn((2, 4, 3), generator=gen, dtype=torch.float64)
    (c * ref.embed_forward(tok, table, 1.7)).sum().backward()
    got, _ = ref.embed_backward(tok, c, 5, 1.7)
    assert torch.allclose(got, table.grad)
