"""GPU check of the embedding gradient where its kernels take other paths: rows wider than one pass over the columns, more
positions than a cluster sorts, tables that are partly cleared during the sort, and one table of all workers added to.  Bounds
as in test_gpu_lm_embed."""
import pytest
import torch

from tests import _lm_reference as ref
from tests.test_gpu_lm_embed import DT, _tokens, backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [2049, 2056, 4102, 5001])
@pytest.mark.parametrize("T", [40, 1500, 4500])
def test_wide_rows(T, D):
    backward(1, T, 30, D, "f32", "bf16", seed=D)
    backward(1, T, 30, D, "bf16", "f32", skew="same", accumulate=True, seed=D + 1)
    backward(2, T // 2, 9, D, "f32", "f32", torch.int32, pads=(8, 3), padding=1, seed=D + 2)


@pytest.mark.parametrize("table", DT)
@pytest.mark.parametrize("act", DT)
@pytest.mark.parametrize("D", [1, 18, 33, 64])
def test_more_positions_than_a_cluster_sorts(table, act, D):
    backward(1, 131073, 5003, D, table, act, seed=D)
    backward(3, 50001, 700, D, table, act, torch.int32, padding=0, accumulate=True, bad=[(0, 0, -1), (2, 50000, 700)], seed=D + 1)


@pytest.mark.parametrize("skew", ["same", "uniform", "zipf"])
@pytest.mark.parametrize("V", [1, 2, 1023, 1024, 300000, 1100000])
def test_tables_of_the_launched_sort(skew, V):
    """One, two and three passes of digits; rows without a token are zeros."""
    backward(1, 140001, V, 4, "f32", "bf16", torch.int32, skew=skew, seed=V)
    backward(2, 70001, V // 2 + 1, 3, "bf16", "f32", skew=skew, padding=0, pads=(1, 2), seed=V + 1)


@pytest.mark.parametrize("T,V", [(9000, 60000), (20000, 60000), (40000, 80000), (70000, 110000)])
@pytest.mark.parametrize("padding", [-1, 0])
def test_tables_that_are_partly_cleared_during_the_sort(T, V, padding):
    """1, 2, 4 and 8 keys a thread, and more rows of 1 KiB than are cleared meanwhile ((6 + T / 4096) 4.5 MB): the others are
    cleared by their flags.  The table holds other values before."""
    assert 0 < (6 + T // 4096) * 4500000 // 1024 < V
    backward(1, T, V, 256, "f32", "bf16", skew="uniform", padding=padding, seed=T)


@pytest.mark.parametrize("T", [1, 60, 2000, 30000, 60000])
@pytest.mark.parametrize("table", DT)
@pytest.mark.parametrize("accumulate", [False, True])
def test_one_table_of_all_workers_added_to(T, table, accumulate):
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(T)
    for V, D in ((90, 48), (2000, 21)):
        P = 3
        tok = _tokens(gen, P, T, V, "zipf")
        d = torch.randn((P, T, D), generator=gen)
        start = torch.randn((V, D), generator=gen).to(DT[table])
        grad = start.cuda()
        lm.Embedding(tok.cuda(), d_out=d.cuda(), d_table=grad[None].expand(P, V, D), accumulate=accumulate, padding=2).backward()
        torch.cuda.synchronize()
        want, size = (t.sum(0) for t in ref.embed_backward(tok, d.double(), V, 1.0, 2))
        if accumulate:
            want, size = want + start.double(), size + start.double().abs()
        counts = torch.bincount(tok.reshape(-1), minlength=V).double()[:, None]
        bound = (counts + 3) * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() if table == "bf16" else 0)
        assert ((grad.cpu().double() - want).abs() <= bound + 1e-38).all()
