"""The oracle of the sequence memory against itself: gradients against differences, a sequence in one piece and in two, what an episode's first
step and a sequence's end cut off."""
import numpy as np
import pytest

import seq_oracle as so

RNG = np.random.default_rng


def scan_case(seed, T=7, N=3, D=4, S=3, G=2):
    r = RNG(seed)
    starts = (r.random((T, N)) < 0.2).astype(np.uint8)
    lengths = np.array([T, 0, T - 2])[:N]
    return dict(x=r.normal(size=(T, N, D)), dt=r.normal(size=(T, N, D)), A=-np.exp(r.normal(size=(D, S))), B=r.normal(size=(T, N, G, S)), C=r.normal(size=(T, N, G, S)),
                z=r.normal(size=(T, N, D)), skip=r.normal(size=D), dt_bias=r.normal(size=D), starts=starts, lengths=lengths, h_in=r.normal(size=(N, D, S)))


@pytest.mark.parametrize("softplus", [True, False])
def test_scan_gradients_are_the_differences(softplus):
    case = dict(scan_case(1), softplus=softplus)
    if not softplus:             # step sizes as they are: none below zero, or states grow
        case["dt"], case["dt_bias"] = np.abs(case["dt"]), np.abs(case["dt_bias"])
    r = RNG(2)
    dy, dh = r.normal(size=case["x"].shape), r.normal(size=case["h_in"].shape)
    value = lambda c: (lambda o: (o["y"] * dy).sum() + (o["h_out"] * dh).sum())(so.scan(**c))  # noqa: E731
    grads = so.scan(**case, dy=dy, dh_out=dh)
    for name, to in (("x", "dx"), ("dt", "ddt"), ("z", "dz"), ("B", "dB"), ("C", "dC"), ("A", "dA"), ("skip", "dskip"), ("dt_bias", "ddt_bias"), ("h_in", "dh_in")):
        way = r.normal(size=case[name].shape)
        e = 1e-6
        up, down = (value({**case, name: case[name] + s * e * way}) for s in (1, -1))
        assert abs((up - down) / (2 * e) - (grads[to] * way).sum()) < 1e-6 * (1 + abs((grads[to] * way).sum())), name


@pytest.mark.parametrize("W,kind", [(2, "silu"), (3, "none"), (4, "silu")])
def test_conv_gradients_are_the_differences(W, kind):
    r = RNG(W)
    T, N, D = 6, 4, 3
    starts, lengths = (r.random((T, N)) < 0.25).astype(np.uint8), np.array([T, 0, 1, T - 2])
    case = dict(x=r.normal(size=(T, N, D)), w=r.normal(size=(D, W)), bias=r.normal(size=D), state=r.normal(size=(N, W - 1, D)))
    dy, ds = r.normal(size=(T, N, D)), r.normal(size=(N, W - 1, D))
    value = lambda c: (lambda o: (o[0] * dy).sum() + (o[1] * ds).sum())(so.conv(**c, starts=starts, lengths=lengths, kind=kind))  # noqa: E731
    grads = so.conv_grad(**case, starts=starts, lengths=lengths, kind=kind, dy=dy, dstate=ds)
    for name, got in zip(("x", "w", "bias", "state"), grads):
        way = r.normal(size=case[name].shape)
        up, down = (value({**case, name: case[name] + s * 1e-6 * way}) for s in (1, -1))
        assert abs((up - down) / 2e-6 - (got * way).sum()) < 1e-6 * (1 + abs((got * way).sum())), name


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
def test_linear_gradients_are_the_differences(kind):
    r = RNG(5)
    x, w, b, res, dy = r.normal(size=(4, 3)), r.normal(size=(5, 3)), r.normal(size=5), r.normal(size=(4, 5)), r.normal(size=(4, 5))
    value = lambda x, w, b: (so.linear(x, w, b, res, kind)[0] * dy).sum()  # noqa: E731
    dx, dw, db = so.linear_grad(x, w, so.linear(x, w, b, res, kind)[1], dy, None, kind)
    for i, got in enumerate((dx, dw, db)):
        args = [x, w, b]
        way = r.normal(size=args[i].shape)
        up, down = (value(*[a + s * 1e-6 * way if k == i else a for k, a in enumerate(args)]) for s in (1, -1))
        assert abs((up - down) / 2e-6 - (got * way).sum()) < 1e-6 * (1 + abs((got * way).sum()))


def test_a_sequence_in_two_pieces():
    case = scan_case(3)
    case["lengths"] = None
    whole = so.scan(**case)
    cut = lambda a, s: {k: v[s] if k in ("x", "dt", "B", "C", "z", "starts") else v for k, v in a.items()}  # noqa: E731
    first = so.scan(**cut(case, slice(0, 3)))
    second = so.scan(**{**cut(case, slice(3, None)), "h_in": first["h_out"]})
    assert np.allclose(np.concatenate([first["y"], second["y"]]), whole["y"], atol=1e-12) and np.allclose(second["h_out"], whole["h_out"], atol=1e-12)
    r = RNG(4)
    x, w, b, st, starts = r.normal(size=(7, 2, 3)), r.normal(size=(3, 4)), r.normal(size=3), r.normal(size=(2, 3, 3)), (r.random((7, 2)) < 0.3).astype(np.uint8)
    y, out, _, _ = so.conv(x, w, b, st, starts, None, "silu")
    for at in (1, 2, 5):
        y1, mid, _, _ = so.conv(x[:at], w, b, st, starts[:at], None, "silu")
        y2, end, _, _ = so.conv(x[at:], w, b, mid, starts[at:], None, "silu")
        assert np.allclose(np.concatenate([y1, y2]), y) and np.allclose(end, out)


def test_what_an_episode_does_not_see():
    case = scan_case(6)
    case["lengths"] = None
    case["starts"][:] = 0
    case["starts"][4] = 1
    changed = {**case, "x": case["x"].copy(), "h_in": case["h_in"] + 5}
    changed["x"][:4] += 3
    a, b = so.scan(**case), so.scan(**changed)
    assert np.array_equal(a["y"][4:], b["y"][4:]) and np.array_equal(a["h_out"], b["h_out"]) and not np.allclose(a["y"][:4], b["y"][:4])
    g = so.scan(**case, dy=np.ones_like(case["x"]), dh_out=np.ones_like(case["h_in"]))
    only_late = so.scan(**case, dy=np.concatenate([np.zeros((4, 3, 4)), np.ones((3, 3, 4))]), dh_out=np.ones_like(case["h_in"]))
    assert not only_late["dx"][:4].any() and not only_late["dh_in"].any() and g["dh_in"].any()


def test_the_count_of_roundings_catches_a_wrong_term():
    case = scan_case(8, T=20)
    case["lengths"] = None
    want, size = so.scan(**case), so.scan(**case, size=True)
    so.near(want["y"].astype(np.float32), want["y"], size["y"], 16 * 20, so.U, "y")
    wrong = {**case, "B": case["B"].copy()}
    wrong["B"][3, 1] = wrong["B"][3, 0]
    with pytest.raises(AssertionError):
        so.near(so.scan(**wrong)["y"].astype(np.float32), want["y"], size["y"], 16 * 20, so.U, "y")
