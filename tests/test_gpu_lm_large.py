"""GPU check of offsets beyond 32 bits: rows, tables and tensors of more than 2^31 values."""
import pytest
import torch

from tests import _lm_reference as ref

pytestmark = pytest.mark.gpu


def _room(gib):
    free, _ = torch.cuda.mem_get_info()
    if free < (gib + 2) << 30:
        pytest.skip(f"needs {gib} GiB")


def test_embedding_rows_far_apart():
    from paper_1905_10395_b200 import lm
    _room(10)
    V, D, ld = 1100, 64, 2_000_000                       # the last row begins at value 2.2e9
    table = torch.zeros(V * ld, dtype=torch.bfloat16, device="cuda")
    view = torch.as_strided(table, (1, V, D), (V * ld, ld, 1))
    view.copy_(torch.randn((1, V, D), device="cuda"))
    for T in (50, 6000):
        tok = torch.randint(0, V, (1, T), device="cuda")
        tok[0, 0] = V - 1
        out = torch.empty((1, T, D), dtype=torch.bfloat16, device="cuda")
        d = torch.randn((1, T, D), device="cuda").to(torch.bfloat16)
        grad = torch.as_strided(table, (1, V, D), (V * ld, ld, 1), D)        # beside the table's own rows
        lm.Embedding(tok, table=view, out=out, d_out=d, d_table=grad).forward()
        op = lm.Embedding(tok, d_out=d, d_table=grad)
        op.backward()
        torch.cuda.synchronize()
        assert torch.equal(out[0], view[0, tok[0]])
        want, size = ref.embed_backward(tok.cpu(), d.cpu().double(), V, 1.0)
        assert ((grad.cpu().double() - want).abs() <= T * 2.0 ** -24 * size + 2.0 ** -8 * want.abs()).all()


def test_norm_rows_far_apart():
    from paper_1905_10395_b200 import lm
    _room(12)
    T, D, ld = 700, 320, 3_200_000                       # the last row begins at value 2.2e9
    buf = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda")
    rows = [torch.as_strided(buf, (1, T, D), (T * ld, ld, 1), k * 1024) for k in range(4)]
    x, y, out, h = rows
    gen = torch.Generator(device="cuda").manual_seed(1)
    for v in (x, y):
        v.copy_(torch.randn((1, T, D), generator=gen, device="cuda"))
    w = torch.ones((1, D), device="cuda")
    near = [torch.empty((1, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lm.BlockNorm(x=x, y=y, w_post=w, w_pre=w, out=out, h=h).forward()
    lm.BlockNorm(x=x.contiguous(), y=y.contiguous(), w_post=w, w_pre=w, out=near[0], h=near[1]).forward()
    torch.cuda.synchronize()
    assert torch.equal(out, near[0]) and torch.equal(h, near[1])
    stats = [torch.rsqrt(v.float().square().mean(-1) + 1e-6) for v in (out, y)]
    far = dict(out=out, y=y, d_out=x, d_h=h, dx=torch.as_strided(buf, (1, T, D), (T * ld, ld, 1), 8192),
               dy=torch.as_strided(buf, (1, T, D), (T * ld, ld, 1), 16384), dw_pre=torch.empty((1, D), device="cuda"),
               dw_post=torch.empty((1, D), device="cuda"))
    close = {k: v.contiguous().clone() for k, v in far.items()}
    for kw in (far, close):
        lm.BlockNorm(w_post=w, w_pre=w, rstd_pre=stats[0], rstd_post=stats[1], **kw).backward()
    torch.cuda.synchronize()
    assert all(torch.equal(far[k], close[k]) for k in ("dx", "dy", "dw_pre", "dw_post"))


def test_adamw_tensor_of_more_than_2_31_values():
    from paper_1905_10395_b200 import lm
    _room(40)
    n, k = 2 ** 31 + 5000, 5000
    p = torch.ones(n, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-k:] = torch.randn(k, device="cuda")
    g[:k] = g[-k:]
    opt = lm.AdamW([p], [g], state="f32", weight_decay=0.1)
    small_p, small_g = torch.ones(k, device="cuda"), g[-k:].clone()
    small = lm.AdamW([small_p], [small_g], state="f32", weight_decay=0.1)
    for o in (opt, small):
        o.step(1e-2)
    torch.cuda.synchronize()
    for lo in (0, n - k):
        assert torch.equal(p[lo:lo + k], small_p)
        assert torch.equal(opt.m[lo:lo + k], small.m[:k]) and torch.equal(opt.v[lo:lo + k], small.v[:k])
    middle = p[k:n - k]
    assert bool((middle == middle[0]).all())
