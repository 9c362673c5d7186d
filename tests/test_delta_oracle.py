"""The oracle of layer norm and of the gated delta rule against differences of itself."""
import numpy as np
import pytest

import delta_oracle as do


def difference(f, x, i, step=1e-6):
    up, down = x.copy(), x.copy()
    up[i] += step
    down[i] -= step
    return (f(up) - f(down)) / (2 * step)


def test_norm():
    r = np.random.default_rng(0)
    x, w, b, dy, add = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7)), r.normal(size=(3, 7))
    out, _ = do.norm(x, w, b, 1e-3, dy, add)
    loss = lambda x, w, b: (do.norm(x, w, b, 1e-3)[0]["y"] * dy).sum() + (x * add).sum()  # noqa: E731
    for i in np.ndindex(3, 7):
        assert abs(difference(lambda v: loss(v, w, b), x, i) - out["dx"][i]) < 1e-7
    for i in range(7):
        assert abs(difference(lambda v: loss(x, v, b), w, i) - out["dw"][i]) < 1e-7 and abs(difference(lambda v: loss(x, w, v), b, i) - out["db"][i]) < 1e-7


@pytest.mark.parametrize("normalize,softplus", [(True, True), (False, False)])
def test_delta(normalize, softplus):
    r = np.random.default_rng(1)
    T, N, G, H, K, V = 6, 2, 2, 4, 3, 2
    given = {"q": r.normal(size=(T, N, G, K)), "k": 0.7 * r.normal(size=(T, N, G, K)), "v": r.normal(size=(T, N, H, V)), "a": 0.3 * r.normal(size=(T, N, H)), "b": r.normal(size=(T, N, H)),
             "A": -0.5 - r.random(H), "a_bias": 0.2 + 0.1 * r.normal(size=H), "h_in": r.normal(size=(N, H, K, V))}
    starts = np.zeros((T, N), dtype=np.uint8)
    starts[3, 1] = 1
    more = {"scale": 0.7, "normalize": normalize, "softplus": softplus, "starts": starts, "lengths": np.array([4, 6])}
    dy, dh = r.normal(size=(T, N, H, V)), r.normal(size=(N, H, K, V))
    out, _ = do.delta(**given, **more, dy=dy, dh_out=dh)

    def loss(**changed):
        o, _ = do.delta(**{**given, **changed}, **more)
        return (o["y"] * dy).sum() + (o["h_out"] * dh).sum()
    for name, x in given.items():
        grad = out["dh_in" if name == "h_in" else "d" + name]
        assert grad.shape == x.shape
        for i in np.ndindex(*x.shape):
            assert abs(difference(lambda v: loss(**{name: v}), x, i) - grad[i]) < 1e-6, (name, i)
