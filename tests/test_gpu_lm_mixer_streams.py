"""The convolution and the scan on streams of their own, captured in CUDA graphs and replayed on new contents, and refused under a
capture that their stream is not part of."""
import pytest
import torch

pytestmark = pytest.mark.gpu

P, T, D, N = 2, 200, 40, 16


def _make(lm, gen, stream=None, ragged=True):
    r = lambda *s: torch.randn(s, generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    f = lambda *s: torch.randn(s, generator=gen).cuda()  # noqa: E731
    ins = {k: r(P, T, D) for k in ("x", "dt", "z", "d_out")} | {k: r(P, T, N) for k in ("b", "c")}
    par = {"a_log": f(P, D, N), "skip": f(P, D), "dt_bias": f(P, D), "w": f(P, D, 4)}
    where = {"starts": torch.tensor([0, 3, 120, 120, 199], dtype=torch.int32, device="cuda")} if ragged else {"sequences": 4}
    out = {k: torch.zeros_like(ins[s]) for k, s in (("v", "x"), ("y", "x"), ("d_x", "x"), ("d_dt", "x"), ("d_z", "x"), ("d_b", "b"), ("d_c", "c"),
                                                    ("dx", "x"))}
    out |= {"d_" + k: torch.zeros_like(v) for k, v in par.items()}
    torch.cuda.synchronize()
    conv = lm.CausalConv(ins["x"], par["w"], out=out["v"], d_out=out["d_x"], dx=out["dx"], dw=out["d_w"], stream=stream, **where)
    scan = lm.SelectiveScan(out["v"], ins["dt"], par["a_log"], ins["b"], ins["c"], z=ins["z"], skip=par["skip"], dt_bias=par["dt_bias"], out=out["y"],
                            d_out=ins["d_out"], d_x=out["d_x"], d_dt=out["d_dt"], d_a_log=out["d_a_log"], d_b=out["d_b"], d_c=out["d_c"],
                            d_z=out["d_z"], d_skip=out["d_skip"], d_dt_bias=out["d_dt_bias"], stream=stream, **where)

    def go():
        conv.forward()
        scan.forward()
        scan.backward()
        conv.backward()
    return ins, out, go


@pytest.mark.parametrize("ragged", [False, True])
def test_captured_and_replayed(ragged):
    from paper_1905_10395_b200 import lm
    s = torch.cuda.Stream()
    ins, out, go = _make(lm, torch.Generator().manual_seed(0), s, ragged)
    go()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go()
    for seed in (1, 2):
        gen = torch.Generator().manual_seed(seed)
        for v in ins.values():
            v.copy_(torch.randn(v.shape, generator=gen))
        for v in out.values():
            v.zero_()
        torch.cuda.synchronize()
        go()
        s.synchronize()
        want = {k: v.clone() for k, v in out.items()}
        for v in out.values():
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.equal(v, want[k]), k
            assert v.abs().sum() > 0, k


def test_two_streams_at_once():
    """Two sets of operators that run at the same time, each with its own scratch, give what each gives alone."""
    from paper_1905_10395_b200 import lm
    sets = [_make(lm, torch.Generator().manual_seed(i), torch.cuda.Stream()) for i in (3, 4)]
    want = []
    for _, out, go in sets:
        go()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in out.items()})
    for _ in range(20):
        for _, _, go in sets:
            go()
    torch.cuda.synchronize()
    for (_, out, _), w in zip(sets, want):
        assert all(torch.equal(v, w[k]) for k, v in out.items())


def test_refused_under_a_capture_of_another_stream():
    from paper_1905_10395_b200 import lm
    mine, other = torch.cuda.Stream(), torch.cuda.Stream()
    _, _, go = _make(lm, torch.Generator().manual_seed(5), mine)
    g = torch.randn(2, 30, 40, device="cuda")
    ortho = lm.Orthogonalize(g, torch.empty_like(g, dtype=torch.bfloat16), stream=mine)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        for call in (go, ortho.forward):
            with pytest.raises(lm.api.LsgdError) as e:
                call()
            assert e.value.status == lm.api.ERR_STATE
        torch.zeros(1, device="cuda")
    torch.cuda.synchronize()


def test_same_inputs_same_bits():
    from paper_1905_10395_b200 import lm
    _, out, go = _make(lm, torch.Generator().manual_seed(6))
    go()
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in out.items()}
    for _ in range(3):
        go()
    torch.cuda.synchronize()
    assert all(torch.equal(v, first[k]) for k, v in out.items())
