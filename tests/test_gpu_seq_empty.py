"""Sequences without steps and steps beyond a sequence's end, whose states are not finite (an idle slot's): nothing of them reaches what the sequences share, the
gradients of their own steps are 0, and their states stay what they are.  Every value is compared with a call whose idle states are finite, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def same(a, b):
    """The same numbers, NaN at the same places."""
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def scan_inputs(T, N, D, S, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    d = {k: normal(T, N, D).to(dtype) for k in ("x", "dt", "z", "dy")}
    d.update({k: normal(T, N, S).to(dtype) for k in ("B", "C")}, A=-torch.exp(normal(D, S)), skip=normal(D), dt_bias=normal(D) - 2, h_in=normal(N, D, S), dh_out=normal(N, D, S))
    return d


def scan(hts, ctx, d, lengths, starts=None, softplus=True):
    T, N, D = d["x"].shape
    like = lambda k: torch.full(d[k].shape, 7.0, dtype=d[k].dtype, device="cuda")  # noqa: E731
    out = dict(y=like("x"), h_out=like("h_in"))
    states = torch.empty(hts.selective_scan_states(T, N, D, d["A"].shape[1]), device="cuda")
    more = dict(z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"], softplus=softplus, starts=starts, lengths=lengths, h_in=d["h_in"])
    ctx.hts_selective_scan(d["x"], d["dt"], d["A"], d["B"], d["C"], out["y"], h_out=out["h_out"], states=states, **more)
    g = {"d" + k: like(k) for k in ("x", "dt", "z", "B", "C", "A", "skip", "dt_bias")}
    g["dh_in"] = like("h_in")
    ctx.hts_selective_scan_backward(d["x"], d["dt"], d["A"], d["B"], d["C"], d["dy"], states, g["dx"], g["ddt"], g["dB"], g["dC"], g["dA"], dz=g["dz"], dskip=g["dskip"], ddt_bias=g["ddt_bias"],
                                    dh_out=d["dh_out"], dh_in=g["dh_in"], **more)
    torch.cuda.synchronize()
    return {**out, **g}


SHAPES = [(40, 4, 20, 16), (1, 3, 70, 16), (33, 5, 130, 13), (700, 3, 24, 8), (300, 4, 18, 33), (9, 3, 16, 64)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,N,D,S", SHAPES)
def test_scan_of_sequences_without_steps(hts, dtype, T, N, D, S):
    d = scan_inputs(T, N, D, S, dtype)
    lengths = torch.tensor([T, 0, max(1, T // 3), 0, T][:N], dtype=torch.int32, device="cuda")
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S, precision=hts.PRECISION_BF16 if dtype is torch.bfloat16 else hts.PRECISION_FP32))
    clean = scan(hts, ctx, d, lengths)
    bad = {**d, "h_in": d["h_in"].clone(), "dh_out": d["dh_out"].clone()}
    idle = [n for n in range(N) if int(lengths[n]) == 0]
    for k, n in enumerate(idle):
        bad["h_in"][n], bad["dh_out"][n] = (INF, NAN) if k % 2 else (NAN, INF)
    bad["h_in"][1, ::2] = -INF
    got = scan(hts, ctx, bad, lengths)
    live = [n for n in range(N) if n not in idle]
    for k, v in got.items():
        if k in ("h_out", "dh_in"):
            want = bad["h_in" if k == "h_out" else "dh_out"]
            assert same(v[idle], want[idle]) and torch.equal(v[live], clean[k][live]), k
        else:
            assert torch.equal(v, clean[k]), k
    for n in range(N):
        for k in ("y", "dx", "ddt", "dz", "dB", "dC"):
            assert bool((got[k][int(lengths[n]):, n] == 0).all()), (k, n)
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,N,D,S", [(40, 4, 20, 16), (33, 2, 130, 13), (700, 3, 24, 8)])
def test_scan_steps_beyond_an_end_that_is_not_finite(hts, dtype, T, N, D, S):
    """The last step of a sequence leaves a state that is not finite, and its gradient is not either: steps beyond it still have gradients of 0, and the states stay."""
    d = scan_inputs(T, N, D, S, dtype)
    ends = [T, T // 2, 5, 17][:N]
    lengths = torch.tensor(ends, dtype=torch.int32, device="cuda")
    d["x"][ends[1] - 1, 1] = INF
    d["dh_out"][1] = NAN
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S, precision=hts.PRECISION_BF16 if dtype is torch.bfloat16 else hts.PRECISION_FP32))
    got = scan(hts, ctx, d, lengths)
    for n in range(N):
        for k in ("y", "dx", "ddt", "dz", "dB", "dC"):
            assert bool((got[k][ends[n]:, n] == 0).all()), (k, n)
    assert not bool(torch.isfinite(got["h_out"][1]).any()) and bool(torch.isfinite(got["dx"][:, [n for n in range(N) if n != 1]]).all())
    ctx.close()


@pytest.mark.parametrize("T", [1, 30, 700])
def test_scan_state_stays_whatever_its_decay(hts, T):
    """A state that forgets at once (A = -inf) is kept, too, where there is no step."""
    N, D, S = 3, 20, 8
    d = scan_inputs(T, N, D, S, torch.float32)
    d["A"][:, 0] = -INF
    lengths = torch.tensor([T, 0, 0], dtype=torch.int32, device="cuda")
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    y, h = torch.empty(T, N, D, device="cuda"), torch.empty(N, D, S, device="cuda")
    ctx.hts_selective_scan(d["x"], d["dt"], d["A"], d["B"], d["C"], y, z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"], lengths=lengths, h_in=d["h_in"], h_out=h)
    torch.cuda.synchronize()
    assert torch.equal(h[1:], d["h_in"][1:]) and bool(torch.isfinite(y).all()) and bool(torch.isfinite(h).all())
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("T,N,D,W", [(40, 4, 20, 4), (1, 3, 72, 4), (17, 5, 33, 3), (8, 3, 64, 2), (3, 4, 128, 4)])
def test_convolution_of_sequences_without_steps(hts, dtype, silu, T, N, D, W):
    g = torch.Generator(device="cuda").manual_seed(T + D)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, dy, w, b, state, dstate = normal(T, N, D).to(dtype), normal(T, N, D).to(dtype), normal(D, W), normal(D), normal(N, W - 1, D), normal(N, W - 1, D)
    lengths = torch.tensor([T, 0, max(1, T // 3), 0, T][:N], dtype=torch.int32, device="cuda")
    idle, live = [n for n in range(N) if int(lengths[n]) == 0], [n for n in range(N) if int(lengths[n])]
    ctx = hts.SeqContext(hts.short_conv_workspace(T, N, D, W))

    def both(state, dstate):
        like = lambda t: torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda")  # noqa: E731
        o = dict(y=like(x), state_out=like(state), dx=like(x), dw=like(w), db=like(b), dstate_in=like(state))
        more = dict(bias=b, act=hts.ACT_SILU if silu else hts.ACT_NONE, lengths=lengths, state_in=state)
        ctx.hts_short_conv(x, w, o["y"], state_out=o["state_out"], **more)
        ctx.hts_short_conv_backward(x, w, dy, o["dx"], o["dw"], db=o["db"], dstate_out=dstate, dstate_in=o["dstate_in"], **more)
        torch.cuda.synchronize()
        return o
    clean, bad, dbad = both(state, dstate), state.clone(), dstate.clone()
    for k, n in enumerate(idle):
        bad[n], dbad[n] = (INF, NAN) if k % 2 else (NAN, INF)
    bad[1, :, ::2] = -INF
    got = both(bad, dbad)
    for k, v in got.items():
        if k in ("state_out", "dstate_in"):
            assert same(v[idle], (bad if k == "state_out" else dbad)[idle]) and torch.equal(v[live], clean[k][live]), k
        else:
            assert torch.equal(v, clean[k]), k
    ctx.close()


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_convolution_beyond_an_end_that_is_not_finite(hts, silu, W):
    """The last inputs of a sequence are NaN: the gradients of the steps beyond it are 0."""
    T, N, D = 29, 3, 40
    x, dy, w, state = (torch.randn(*s, device="cuda") for s in ((T, N, D), (T, N, D), (D, W), (N, W - 1, D)))
    ends = [T, 11, 16]
    x[ends[1] - 2:ends[1], 1], x[ends[2] - 1, 2] = NAN, INF
    dx, dw = torch.full((T, N, D), 7.0, device="cuda"), torch.empty(D, W, device="cuda")
    ctx = hts.SeqContext(hts.short_conv_workspace(T, N, D, W))
    ctx.hts_short_conv_backward(x, w, dy, dx, dw, act=hts.ACT_SILU if silu else hts.ACT_NONE, lengths=torch.tensor(ends, dtype=torch.int32, device="cuda"), state_in=state,
                                dstate_out=torch.randn(N, W - 1, D, device="cuda"))
    torch.cuda.synchronize()
    for n in range(N):
        assert bool((dx[ends[n]:, n] == 0).all()), n
    assert bool(torch.isfinite(dx[:, 0]).all())
    ctx.close()
