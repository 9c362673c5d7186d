"""The operators of the sequence memory in binary64, step by step from their definitions (numpy, no code of the package), and how far a
binary32 computation may be from them.

Every function also runs with `size=True`: the same sums with every term by its absolute value.  A sum of n rounded terms in any order is
within about n u of the sum of the terms' sizes, u = 2^-24, so an output may differ by its own rounding (half a step) and a count of
roundings times u times that size.
"""
import math

import numpy as np

U = 2.0 ** -24


def erf(v):
    return np.vectorize(math.erf, otypes=[float])(v)


def sigmoid(v):
    with np.errstate(over="ignore"):
        return np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))


def act(v, kind):
    return {"none": lambda: v, "relu": lambda: np.maximum(v, 0), "silu": lambda: v * sigmoid(v), "gelu": lambda: v * 0.5 * (1 + erf(v / math.sqrt(2)))}[kind]()


def slope(v, kind, size=False):
    if kind == "none":
        return np.ones_like(v)
    if kind == "relu":
        return (v > 0).astype(float)
    w = np.abs(v) if size else v
    if kind == "silu":
        s = sigmoid(v)
        return s * (1 + w * (1 - s))
    return 0.5 * (1 + erf(v / math.sqrt(2))) + w * np.exp(-v * v / 2) / math.sqrt(2 * math.pi)


def linear(x, w, bias, residual, kind, size=False):
    f = np.abs if size else (lambda a: a)
    pre = f(x) @ f(w).T + (0 if bias is None else f(bias))
    y = pre if size else act(pre, kind)
    return (y if residual is None else y + f(residual)), pre


def linear_grad(x, w, pre, dy, add, kind, size=False):
    f = np.abs if size else (lambda a: a)
    g = f(dy) * (1 if kind == "none" else slope(pre, kind, size))
    return g @ f(w) + (0 if add is None else f(add)), g.T @ f(x), g.sum(0)


def _length(lengths, n, T):
    return T if lengths is None else max(0, min(T, int(lengths[n])))


def conv(x, w, bias, state, starts, lengths, kind):
    """y, state_out, and the steps' pre-activations and the inputs (step number or -1, -2 .. for the state's) that each saw."""
    T, N, D = x.shape
    W = w.shape[1]
    y, pre, out, seen = np.zeros_like(x), np.zeros_like(x), np.zeros((N, W - 1, D)), {}
    for n in range(N):
        # input number i: state for i < 0 (state[W - 1 + i]), x otherwise
        value = lambda i: (0 * w[:, 0] if state is None else state[n, W - 1 + i]) if i < 0 else x[i, n]  # noqa: E731
        reach, length = -(W - 1), _length(lengths, n, T)
        for t in range(length):
            if starts is not None and starts[t, n]:
                reach = t
            taps = [(j, t - W + 1 + j) for j in range(W) if t - W + 1 + j >= reach]
            seen[t, n] = taps
            pre[t, n] = (0 if bias is None else bias) + sum(w[:, j] * value(i) for j, i in taps)
            y[t, n] = act(pre[t, n], kind)
        for j in range(W - 1):
            i = length - (W - 1) + j
            out[n, j] = value(i) if i >= reach else 0
        seen["reach", n] = reach
    return y, out, pre, seen


def conv_grad(x, w, bias, state, starts, lengths, kind, dy, dstate, size=False):
    T, N, D = x.shape
    W = w.shape[1]
    _, _, pre, seen = conv(x, w, bias, state, starts, lengths, kind)
    f = np.abs if size else (lambda a: a)
    dx, dw, db, din = np.zeros_like(x), np.zeros_like(w), np.zeros(D), np.zeros((N, W - 1, D))

    def give(i, n, v):
        if i < 0:
            din[n, W - 1 + i] += v
        else:
            dx[i, n] += v
    for n in range(N):
        length = _length(lengths, n, T)
        for t in range(length):
            g = f(dy[t, n]) * slope(pre[t, n], kind, size)
            db += g
            for j, i in seen[t, n]:
                value = (0 * db if state is None else state[n, W - 1 + i]) if i < 0 else x[i, n]
                dw[:, j] += g * f(value)
                give(i, n, g * f(w[:, j]))
        for j in range(W - 1):
            i = length - (W - 1) + j
            if dstate is not None and i >= seen["reach", n]:
                give(i, n, f(dstate[n, j]))
    return dx, dw, db, din


def scan(x, dt, A, B, C, z=None, skip=None, dt_bias=None, softplus=True, starts=None, lengths=None, h_in=None, dy=None, dh_out=None, size=False):
    """A dict of the outputs; with dy the gradients too."""
    f = np.abs if size else (lambda a: a)
    T, N, D = x.shape
    G, S = B.shape[2:]
    group = np.arange(D) // (D // G)
    v = dt + (0 if dt_bias is None else dt_bias)
    step = np.logaddexp(0, v) if softplus else v
    rise = sigmoid(v) if softplus else np.ones_like(v)
    gate = np.ones_like(x) if z is None else z * sigmoid(z)
    k = np.zeros(D) if skip is None else skip
    h = np.zeros((N, D, S)) if h_in is None else f(h_in).astype(float)
    out = {"y": np.zeros_like(x)}
    kept, raws = {}, np.zeros_like(x)
    h = h.copy()
    for t in range(T):
        for n in range(N):
            if t >= _length(lengths, n, T):
                continue
            begin = starts is not None and bool(starts[t, n])
            a = np.exp(step[t, n][:, None] * A)
            past = np.zeros((D, S)) if begin else a * h[n]
            b, c = f(B[t, n][group]), f(C[t, n][group])
            h[n] = past + f(step[t, n] * x[t, n])[:, None] * b
            raws[t, n] = (h[n] * c).sum(1) + f(k * x[t, n])
            out["y"][t, n] = raws[t, n] * f(gate[t, n])
            kept[t, n] = (a, past, h[n].copy(), begin)
    out["h_out"] = h
    if dy is None:
        return out
    g = np.zeros((N, D, S)) if dh_out is None else f(dh_out).astype(float).copy()
    for name in ("dx", "ddt", "dz"):
        out[name] = np.zeros_like(x)
    out["dB"], out["dC"], out["dA"], out["dskip"] = np.zeros_like(B), np.zeros_like(B), np.zeros((D, S)), np.zeros(D)
    for t in reversed(range(T)):
        for n in range(N):
            if (t, n) not in kept:
                continue
            a, past, now, begin = kept[t, n]
            r = f(dy[t, n] * gate[t, n])
            b, c = f(B[t, n][group]), f(C[t, n][group])
            gt = r[:, None] * c + g[n]
            np.add.at(out["dB"][t, n], group, gt * f(step[t, n] * x[t, n])[:, None])
            np.add.at(out["dC"][t, n], group, r[:, None] * now)
            gb = (gt * b).sum(1)
            out["dx"][t, n] = gb * f(step[t, n]) + r * f(k)
            out["ddt"][t, n] = ((gt * past * f(A)).sum(1) + gb * f(x[t, n])) * rise[t, n]
            if z is not None:
                out["dz"][t, n] = f(dy[t, n]) * raws[t, n] * f(slope(z[t, n], "silu", size))
            out["dA"] += gt * past * f(step[t, n])[:, None]
            out["dskip"] += r * f(x[t, n])
            g[n] = 0 if begin else a * gt
    out["ddt_bias"], out["dh_in"] = out["ddt"].sum((0, 1)), g
    return out


def near(got, want, size, roundings, half_step, name=""):
    """Every entry within its own rounding and `roundings` roundings of binary32 of the sum of its terms' sizes."""
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    allowed = half_step * np.abs(want) * (1 + 1e-6) + roundings * U * size + 1e-37
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want)
    bad = ~(off <= allowed)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off / allowed)), off.shape)
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} entries off; at {i} got {got[i]!r}, want {want[i]!r}, allowed {allowed[i]:.3e}")
