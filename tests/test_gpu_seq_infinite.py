"""Infinities within the scan's sequences, where every number is positive so that the formula gives infinities and never NaN: what only the kernels have (states
beyond S, channels beyond the last, segments) must not turn them into NaN."""
import pytest
import torch

from test_gpu_seq_empty import scan

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def positive(T, N, D, S, seed=2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    some = lambda *s: torch.rand(*s, device="cuda", generator=g) + 0.25  # noqa: E731
    d = {k: some(T, N, D) for k in ("x", "dt", "z", "dy")}
    d.update({k: some(T, N, S) for k in ("B", "C")}, A=-some(D, S) * 0.05, skip=some(D), dt_bias=some(D) - 3, h_in=some(N, D, S), dh_out=some(N, D, S))
    return d


SHAPES = [(1, 2, 20, 3), (7, 2, 20, 13), (40, 1, 37, 20), (33, 2, 16, 33), (700, 1, 20, 5), (50, 2, 30, 16)]


@pytest.mark.parametrize("T,N,D,S", SHAPES)
def test_an_infinite_step_size(hts, T, N, D, S):
    d = positive(T, N, D, S)
    at = T // 2
    d["dt"][at, 0, 3] = INF
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    got = scan(hts, ctx, d, None)
    # delta x B is infinite from there on, the state before it counts nothing
    want = torch.zeros(T, N, D, dtype=torch.bool, device="cuda")
    want[at:, 0, 3] = True
    assert torch.equal(got["y"] == INF, want) and not bool(torch.isnan(got["y"]).any())
    assert bool((got["h_out"][0, 3] == INF).all()) and not bool(torch.isnan(got["h_out"]).any())
    # C's gradient at those steps is the sum over the channels of r h, infinite; B's are r times factors that end there
    assert bool((got["dC"][at:, 0] == INF).all()) and bool(torch.isfinite(got["dC"][:at, 0]).all()) and bool(torch.isfinite(got["dC"][:, 1:]).all())
    ctx.close()


@pytest.mark.parametrize("T,N,D,S", SHAPES)
def test_an_infinite_gradient(hts, T, N, D, S):
    d = positive(T, N, D, S)
    at = T // 2
    d["dy"][at, 0, 3] = INF
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    got = scan(hts, ctx, d, None)
    want = torch.zeros(T, N, D, dtype=torch.bool, device="cuda")
    want[:at + 1, 0, 3] = True
    assert torch.equal(got["dx"] == INF, want) and not bool(torch.isnan(got["dx"]).any())
    assert bool((got["dB"][:at + 1, 0] == INF).all()) and not bool(torch.isnan(got["dB"]).any())
    assert bool((got["dC"][at, 0] == INF).all()) and not bool(torch.isnan(got["dC"]).any())
    assert bool((got["dh_in"][0, 3] == INF).all()) and not bool(torch.isnan(got["dh_in"]).any())
    ctx.close()


@pytest.mark.parametrize("T,N,D,S", SHAPES)
@pytest.mark.parametrize("which", ["B", "C"])
def test_an_infinite_entry_of_B_or_C(hts, T, N, D, S, which):
    """Of one state at one step: C's gradient of that state is infinite from there on for B, B's up to there for C."""
    d = positive(T, N, D, S)
    at = T // 2
    d[which][at, 0, S - 1] = INF
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    got = scan(hts, ctx, d, None)
    for k in ("dB", "dC"):
        want = torch.zeros(T, N, S, dtype=torch.bool, device="cuda")
        if k[1] != which:
            want[slice(at, T) if which == "B" else slice(0, at + 1), 0, S - 1] = True
        assert torch.equal(got[k] == INF, want) and not bool(torch.isnan(got[k]).any()), k
    ctx.close()
