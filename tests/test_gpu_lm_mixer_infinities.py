"""Infinities in the scan: what stands in for states that do not exist (up to 4, 8, 16, 32 or 64), for channels behind the last and for
rows of no sequence is not multiplied by them.  All values are positive, so that the definition gives infinities, not NaN."""
import pytest
import torch

from tests import _lm_mixer_reference as ref

pytestmark = pytest.mark.gpu


def _run(T, D, N, where, S=1, starts=None, rates=-2.0, seed=0, grads=True):
    from paper_1905_10395_b200 import lm
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.rand(s, generator=gen) * 0.5 + 0.25  # noqa: E731
    host = {"x": r(1, T, D), "dt": r(1, T, D), "b": r(1, T, N), "c": r(1, T, N), "z": r(1, T, D), "a_log": r(1, D, N) + rates}
    for k, at in where.items():
        host[k][0, at[0], at[1]] = float("inf")
    up = r(1, T, D)
    dev = {k: v.cuda() for k, v in host.items()}
    out = {"out": torch.zeros_like(dev["x"])}
    state = torch.full((1, S, D, N), 0.5, device="cuda") if not grads else None
    if grads:
        out |= {"d_" + k: torch.zeros_like(v) for k, v in dev.items()}
    op = lm.SelectiveScan(dev["x"], dev["dt"], dev["a_log"], dev["b"], dev["c"], z=dev["z"], state=state,
                          d_out=up.cuda() if grads else None, sequences=None if starts is not None else S,
                          starts=starts.cuda() if starts is not None else None, **out)
    op.forward()
    if grads:
        op.backward()
    torch.cuda.synchronize()
    edges = ref.edges_of(1, T, S, starts)
    f = {k: v.double() for k, v in host.items()}
    got, size = ref.scan(f["x"], f["dt"], f["a_log"], f["b"], f["c"], f["z"], None, None, None if grads else torch.full((1, S, D, N), 0.5, dtype=torch.float64),
                         up.double() if grads else None, edges)
    if state is not None:
        out["state"] = state
    rel = 2 * (T + D + 64) * 2.0 ** -22                                # test_gpu_lm_scan.py
    for k, v in out.items():
        mine, want, mag = v.double().cpu(), got[k], size[k]
        if k not in ("d_a_log", "state"):                               # rows of no sequence are NaN in the definition's results
            live = torch.zeros(T, dtype=torch.bool)
            live[edges[0][0]:edges[0][-1]] = True
            mine, want, mag = mine[:, live], want[:, live], mag[:, live]
        if "c" in where and k in ("d_a_log", "d_dt"):
            # h in front of a sequence is the constant zero: no gradient passes through it, which the restatement's 0 times an infinite g
            # does not show (its first row's d_dt, and so the whole of d_a_log)
            if k == "d_a_log":
                continue
            first = torch.tensor([lo - edges[0][0] for lo, hi in zip(edges[0], edges[0][1:]) if hi > lo])
            mine, want, mag = (v.index_fill(1, first, 0.0) for v in (mine, want, mag))
        odd = ~torch.isfinite(want)
        same = (mine == want) | (torch.isnan(mine) & torch.isnan(want))
        assert same[odd].all(), f"{k}: {want[odd & ~same][:4]} is {mine[odd & ~same][:4]}"
        close = ~odd & (mag < 1e300)
        assert ((mine - want).abs() <= rel * mag + 1e-35)[close].all(), k
        assert torch.isfinite(mine[~odd]).all(), k
    assert not torch.isfinite(got["out"]).all() or not where, "the case holds no infinity"


@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 11, 13, 16, 20, 33, 64])
def test_an_infinite_input(N):
    _run(40, 24, N, {"x": (7, 3)}, seed=N)
    _run(40, 24, N, {"dt": (7, 3)}, seed=N)


@pytest.mark.parametrize("N", [1, 3, 13, 16])
@pytest.mark.parametrize("what", ["b", "c"])
def test_an_infinite_row_of_b_or_c(N, what):
    """Every channel's sums hold it; 24 and 21 channels leave some of a block without one."""
    for D in (24, 21):
        _run(40, D, N, {what: (7, slice(None))}, seed=N)


@pytest.mark.parametrize("N", [1, 3, 13])
def test_single_tokens_and_split_rows(N):
    _run(30, 9, N, {"x": (7, 3)}, S=30, grads=False, seed=N)
    _run(30, 9, N, {"dt": (7, 3)}, S=30, grads=False, seed=N)
    _run(300, 9, N, {"x": (280, 3)}, rates=-6.0, seed=N)


@pytest.mark.parametrize("starts", [[0, 20, 37], [3, 20, 37]], ids=str)
def test_rows_behind_the_last_sequence(starts):
    """What a sequence ends with, infinite, does not meet the rows of no sequence that share its tile."""
    _run(40, 24, 16, {"x": (30, 3)}, S=2, starts=torch.tensor(starts, dtype=torch.int32), seed=5)


@pytest.mark.parametrize("T,starts", [(20, None), (32, None), (40, [0, 20, 37]), (300, None), (300, [3, 100, 290])], ids=str)
def test_states_that_forget_at_once(T, starts):
    """exp(a_log) beyond fp32: a decay of zero; the definition's results are finite, whatever rows share a tile with the last one."""
    S = 1 if starts is None else len(starts) - 1
    _run(T, 24, 16, {}, S=S, starts=None if starts is None else torch.tensor(starts, dtype=torch.int32), rates=95.0, seed=T)


def test_single_tokens_that_forget_at_once():
    _run(30, 9, 3, {}, S=30, grads=False, rates=95.0)
