"""GPU check of the embedding lookup and its gradient (lsgd_embed_*) against their 64-bit restatement.

Bounds.  The lookup is one fp32 product, rounded to nearest where it is stored in bf16: its bits are known.  A row of the
gradient adds n terms in fp32, at most n 2^-24 of the sum of their magnitudes off, and is scaled and rounded once (by at most
2^-8 of the value in bf16)."""
import pytest
import torch

from tests import _lm_reference as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _tokens(gen, P, T, V, skew):
    if skew == "same":
        return torch.full((P, T), V // 2, dtype=torch.int64)
    u = torch.rand((P, T), generator=gen, dtype=torch.float64)
    if skew == "zipf":
        return (torch.exp(u * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))) - 1).floor().clamp(0, V - 1).long()
    return (u * V).floor().clamp(0, V - 1).long()


def forward(P, T, V, D, table="f32", act="f32", index=torch.int64, pads=(0, 0), offset=0, seed=0, interleaved=False, scale=3.7):
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(seed)
    tok = _tokens(gen, P, T, V, "zipf")
    tab = torch.randn((P, V, D), generator=gen, dtype=torch.float64).to(DT[table])
    g_tab = ref.Guarded((P, V, D), (V * (D + pads[0]), D + pads[0], 1), DT[table], offset, tab)
    st = (D + pads[1], P * (D + pads[1]), 1) if interleaved else (T * (D + pads[1]), D + pads[1], 1)
    out = ref.Guarded((P, T, D), st, DT[act], offset)
    lm.Embedding(tok.to(index).cuda(), table=g_tab.view, out=out.view, scale=scale).forward()
    torch.cuda.synchronize()
    # the product of two fp32 numbers is exact in 64 bits: rounded to fp32, then to the output's type
    want = ref.embed_forward(tok, tab.double(), float(torch.tensor(scale))).float().to(DT[act])
    assert torch.equal(out.view.cpu(), want)
    assert out.intact() and g_tab.intact()


def backward(P, T, V, D, table="f32", act="f32", index=torch.int64, skew="zipf", padding=-1, accumulate=False, pads=(0, 0), offset=0,
             seed=0, scale=0.37, bad=()):
    from paper_1905_10395_b200 import api, lm
    gen = torch.Generator().manual_seed(seed)
    tok = _tokens(gen, P, T, V, skew)
    for p, t, v in bad:
        tok[p, t] = v
    d = torch.randn((P, T, D), generator=gen, dtype=torch.float64).to(DT[act])
    start = torch.randn((P, V, D), generator=gen, dtype=torch.float64).to(DT[table])
    g_out = ref.Guarded((P, T, D), (T * (D + pads[1]), D + pads[1], 1), DT[act], offset, d)
    g_tab = ref.Guarded((P, V, D), (V * (D + pads[0]), D + pads[0], 1), DT[table], offset, start)
    op = lm.Embedding(tok.to(index).cuda(), d_out=g_out.view, d_table=g_tab.view, scale=scale, padding=padding, accumulate=accumulate)
    op.backward()
    torch.cuda.synchronize()
    want, size = ref.embed_backward(tok, d.double(), V, float(torch.tensor(scale)), padding)
    if accumulate:
        want, size = want + start.double(), size + start.double().abs()
    counts = torch.stack([torch.bincount(t[(t >= 0) & (t < V)], minlength=V) for t in tok]).double()[..., None]
    bound = (counts + 3) * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() if table == "bf16" else 0)
    got = g_tab.view.cpu().double()
    assert ((got - want).abs() <= bound + 1e-38).all(), ((got - want).abs() - bound).max()
    if not accumulate:
        assert (got[(counts == 0).expand_as(got)] == 0).all()
    assert g_out.intact() and g_tab.intact()
    assert api.lsgd_embed_check_device() == (api.DEVFLAG_BAD_INDEX if bad else 0)
    return op, g_tab


@pytest.mark.parametrize("table", DT)
@pytest.mark.parametrize("act", DT)
@pytest.mark.parametrize("D", [1, 2, 7, 8, 64, 250, 256, 1000, 1024, 2056, 5001])
def test_lookup_rows_and_types(table, act, D):
    forward(2, 37, 50, D, table, act, seed=D)
    forward(1, 9, 11, D, table, act, torch.int32, pads=(3, 5), offset=1, seed=D)
    forward(3, 5, 20, D, table, act, torch.int32, pads=(8, 16), interleaved=True, seed=D)


@pytest.mark.parametrize("T", [0, 1, 2, 3, 4, 5, 511, 3000])
def test_lookup_lengths(T):
    for P, V, D in ((1, 1, 8), (2, 1000, 96), (1, 7, 2050)):
        forward(P, T, V, D, "f32", "bf16", seed=T)


def test_lookup_shared_table_and_bad_tokens():
    from paper_1905_10395_b200 import api, lm
    gen = torch.Generator().manual_seed(3)
    V, D = 30, 72
    tab = torch.randn((V, D), generator=gen)
    tok = torch.randint(0, V, (3, 10), generator=gen)
    tok[0, 0], tok[2, 9], tok[1, 4] = -1, V, 2 ** 40
    out = torch.full((3, 10, D), float("nan"), device="cuda")
    lm.Embedding(tok.cuda(), table=tab.cuda()[None].expand(3, V, D), out=out).forward()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().double(), ref.embed_forward(tok, tab.double()[None].expand(3, V, D), 1.0))
    assert api.lsgd_embed_check_device() == api.DEVFLAG_BAD_INDEX
    assert api.lsgd_embed_check_device() == 0


@pytest.mark.parametrize("table", DT)
@pytest.mark.parametrize("act", DT)
@pytest.mark.parametrize("T", [40, 1500, 4500])         # few tokens: one launch; more: sorted
@pytest.mark.parametrize("D", [1, 2, 8, 63, 250, 256, 264, 1032])
def test_gradient_rows_and_types(table, act, T, D):
    backward(1, T, 300, D, table, act, seed=D)
    backward(2, T, 77, D, table, act, torch.int32, padding=0, accumulate=True, seed=D + 1)
    backward(1, T, 40, D, table, act, pads=(3, 5), offset=1, padding=3, seed=D + 2)


@pytest.mark.parametrize("T", [0, 1, 2, 31, 32, 33, 1023, 1024, 1025, 2048, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16385, 40000, 65536, 65537, 70001,
                               140000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_lengths(T, accumulate):
    backward(1, T, 1009, 16, "f32", "bf16", accumulate=accumulate, seed=T)
    if T <= 33000:
        backward(2, T, 1, 8, "f32", "f32", accumulate=accumulate, skew="same", seed=T)


@pytest.mark.parametrize("skew", ["same", "uniform", "zipf"])
@pytest.mark.parametrize("V", [1, 2, 3, 255, 256, 511, 512, 513, 70000, 300000])
def test_gradient_tables(skew, V):
    for T in (300, 5000, 66000):
        backward(1, T, V, 8, "f32", "f32", torch.int32, skew=skew, seed=V)
    backward(3, 2500, V, 40, "bf16", "bf16", skew=skew, padding=0, seed=V + 1)


def test_all_tokens_are_padding():
    for T in (5, 4000):
        backward(2, T, 10, 24, skew="same", padding=5)
        backward(2, T, 10, 24, skew="same", padding=5, accumulate=True)


def test_bad_tokens_add_to_nothing():
    for T in (100, 3000):
        backward(2, T, 50, 32, bad=[(0, 0, -1), (1, T - 1, 50), (0, 7, 2 ** 33)], seed=T)
        backward(2, T, 50, 32, torch.float32 and "f32", "bf16", bad=[(0, 3, -(2 ** 62))], padding=1, seed=T)


def test_one_table_of_all_workers():
    """d_table expanded over the workers: the gradient of a shared table is the sum over them."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(4)
    for T in (60, 2000):
        P, V, D = 3, 90, 48
        tok = _tokens(gen, P, T, V, "zipf")
        d = torch.randn((P, T, D), generator=gen)
        grad = torch.full((V, D), 7.0, device="cuda")
        lm.Embedding(tok.cuda(), d_out=d.cuda(), d_table=grad[None].expand(P, V, D)).backward()
        torch.cuda.synchronize()
        want, size = ref.embed_backward(tok, d.double(), V, 1.0)
        want, size = want.sum(0), size.sum(0)
        assert ((grad.cpu().double() - want).abs() <= P * T * 2.0 ** -24 * size).all()


def test_same_inputs_same_bits():
    from paper_1905_10395_b200 import lm
    gen = torch.Generator(device="cuda").manual_seed(5)
    for T in (900, 30000, 90000):
        tok = (torch.rand((1, T), generator=gen, device="cuda").pow(6) * 500).long()
        d = torch.randn((1, T, 64), generator=gen, device="cuda")
        got = []
        for _ in range(3):
            g = torch.empty((1, 500, 64), device="cuda")
            lm.Embedding(tok, d_out=d, d_table=g).backward()
            got.append(g)
        torch.cuda.synchronize()
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_scratch_is_free_and_the_op_repeats():
    """What the scratch holds at the call plays no part, and a bound operator may be called again with new values."""
    gen = torch.Generator().manual_seed(6)
    for T in (5000, 70000):
        op, tab = backward(1, T, 400, 24, seed=1)
        first = tab.view.clone()
        op._keep[1].fill_(255)
        op.backward()
        torch.cuda.synchronize()
        assert torch.equal(first, tab.view)


def test_gradient_against_differences():
    """The loss sum(c out) is linear in the table: its difference along a direction is the gradient's product with it."""
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(7)
    for T in (50, 2000):
        V, D = 40, 33
        tok = _tokens(gen, 2, T, V, "zipf")
        table, u = (torch.randn((2, V, D), generator=gen, dtype=torch.float64) for _ in range(2))
        c = torch.randn((2, T, D), generator=gen, dtype=torch.float64).float()
        grad = torch.empty((2, V, D), device="cuda")
        lm.Embedding(tok.cuda(), d_out=c.cuda(), d_table=grad, scale=2.0).backward()
        torch.cuda.synchronize()
        loss = lambda t: float((c.double() * ref.embed_forward(tok, t, 2.0)).sum())  # noqa: E731
        num = (loss(table + u) - loss(table - u)) / 2
        mine = grad.cpu().double() * u
        assert abs(num - float(mine.sum())) <= 1e-5 * float(mine.abs().sum())


def test_captured_in_a_graph():
    from paper_1905_10395_b200 import lm
    gen = torch.Generator(device="cuda").manual_seed(8)
    tok = torch.randint(0, 300, (1, 5000), generator=gen, device="cuda")
    d = torch.randn((1, 5000, 64), generator=gen, device="cuda")
    want, got = (torch.empty((1, 300, 64), device="cuda") for _ in range(2))
    lm.Embedding(tok, d_out=d, d_table=want).backward()
    s = torch.cuda.Stream()
    op = lm.Embedding(tok, d_out=d, d_table=got, stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        op.backward()
    d.mul_(2.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, 2 * want)
