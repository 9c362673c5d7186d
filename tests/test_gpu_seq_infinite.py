"""Infinities within the scan's sequences, where every number is positive so that the formula gives infinities and never NaN: what only the kernels have (states
beyond S, channels beyond the last, segments) must not turn them into NaN."""
import numpy as np
import pytest
import torch

import seq_oracle as so
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


@pytest.mark.parametrize("S", [5, 16])
@pytest.mark.parametrize("T", [60, 700])
def test_decays_over_one(hts, T, S):
    """Negative step sizes grow a state: from nothing it stays nothing, however large the factors' product, and a small one that a segment's factors take beyond
    binary32's range and the next ones back is what it is step by step."""
    N, D = 1, 24
    d = positive(T, N, D, S)
    d["dt_bias"] = None
    d["A"] = -torch.ones(D, S, device="cuda")
    d["dt"].fill_(-3.5)
    d["x"].zero_()
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    y, h = torch.empty(T, N, D, device="cuda"), torch.empty(N, D, S, device="cuda")
    ctx.hts_selective_scan(d["x"], d["dt"], d["A"], d["B"], d["C"], y, z=d["z"], skip=d["skip"], softplus=False, h_out=h)
    torch.cuda.synchronize()
    assert bool((y == 0).all()) and bool((h == 0).all())
    d["dt"][32:] = 3.5
    small = torch.full((N, D, S), 1e-30, device="cuda")
    ctx.hts_selective_scan(d["x"], d["dt"], d["A"], d["B"], d["C"], y, z=d["z"], skip=d["skip"], softplus=False, h_in=small, h_out=h)
    torch.cuda.synchronize()
    wide = {k: v.double().cpu().numpy() for k, v in d.items() if k not in ("dy", "dh_out", "h_in", "dt_bias")}
    wide["B"], wide["C"] = wide["B"][:, :, None], wide["C"][:, :, None]
    want = so.scan(**wide, softplus=False, h_in=small.double().cpu().numpy())
    # a step's roundings and its exponent's; a segment's product is of one exponent, at most 112 / log 2 of it, rounded once and to 2^-24 of itself
    so.near(y.double().cpu().numpy(), want["y"], np.abs(want["y"]), 16 * (min(T, 64) + S) + 12 * 112, 2.0 ** -24, "y")
    ctx.close()


def test_an_infinite_state_stays(hts):
    """A state that is infinite decays by less than everything at every step, so it stays infinite, however many steps a segment has."""
    T, N, D, S = 700, 1, 24, 8
    d = positive(T, N, D, S)
    d["A"], d["dt_bias"] = torch.full((D, S), -5.0, device="cuda"), torch.zeros(D, device="cuda")
    d["h_in"][0, 5] = INF
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    got = scan(hts, ctx, d, None)
    assert bool((got["y"][:, 0, 5] == INF).all()) and bool((got["h_out"][0, 5] == INF).all())
    rest = [k for k in range(D) if k != 5]
    assert bool(torch.isfinite(got["y"][:, :, rest]).all()) and bool(torch.isfinite(got["h_out"][:, rest]).all())
    ctx.close()


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("W", [2, 4])
def test_an_infinite_filter_weight(hts, silu, W):
    """The weight of the oldest input, infinite for one channel: steps that do not see that input, at an episode's beginning, are what they are without it, and so are the
    other channels; forward and backward."""
    T, N, D = 21, 2, 40
    g = torch.Generator(device="cuda").manual_seed(W)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, dy, w, b, state = normal(T, N, D), normal(T, N, D), normal(D, W), normal(D), normal(N, W - 1, D)
    starts = torch.zeros(T, N, dtype=torch.uint8, device="cuda")
    starts[0], starts[9, 0], starts[20, 1] = 1, 1, 1
    ctx = hts.SeqContext(hts.short_conv_workspace(T, N, D, W))
    unseen = torch.zeros(T, N, dtype=torch.bool, device="cuda")
    for t, n in ((0, 0), (0, 1), (9, 0), (20, 1)):
        unseen[t:t + W - 1, n] = True
    more = dict(bias=b, act=hts.ACT_SILU if silu else hts.ACT_NONE, starts=starts, state_in=state)
    results = []
    for weight in (0.5, INF):
        w[7, 0] = weight
        y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
        ctx.hts_short_conv(x, w, y, **more)
        # only steps that do not see the oldest input have a gradient
        ctx.hts_short_conv_backward(x, w, dy * unseen[:, :, None], dx, dw, **more)
        torch.cuda.synchronize()
        results.append((y, dx, dw))
    (y, dx, dw), (y2, dx2, dw2) = results
    rest = [d for d in range(D) if d != 7]
    assert torch.equal(y[unseen], y2[unseen]) and torch.equal(y[:, :, rest], y2[:, :, rest])
    assert silu or not bool(torch.isfinite(y2[~unseen][:, 7]).any())          # (silu of -inf is 0)
    assert torch.equal(dx[:, :, rest], dx2[:, :, rest]) and torch.equal(dw[rest], dw2[rest])
    # channel 7: what no step beyond the beginnings reaches, whose gradients are 0 times an infinite weight or slope
    assert torch.equal(dx[20, 1, 7], dx2[20, 1, 7])
    ctx.close()
