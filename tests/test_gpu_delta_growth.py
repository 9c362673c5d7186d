"""The gated delta rule where steps lengthen the state, over long sequences that are worked on in segments: what a segment makes of the state before it may be beyond binary32
while every state is within it, and a state of nothing stays nothing."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from test_gpu_delta_rule import Case
from test_gpu_seq import HALF, hts, host, put  # noqa: F401

pytestmark = pytest.mark.gpu


def grown(c, a):
    """The decays' logarithms as they are (A = 1, no softplus), exactly representable in both types."""
    T, N, _, H, _, _ = c.shape
    c.at["A"], c.wide["A"] = put(np.ones(H))
    c.at["a"], c.wide["a"] = put(np.broadcast_to(a[:, None, None], (T, N, H)), c.ty)


def alone_and_beside_others(hts, c, many):  # noqa: F811
    """The same sequence in segments and, as one of many, without them."""
    T, _, G, H, K, V = c.shape
    one = c.run(False)
    other = Case(hts, c.dtype, T, many, G, H, K, V, softplus=False, normalize=c.more["normalize"], state=c.at["h_in"] is not None)
    for name in ("q", "k", "v", "a", "b"):
        other.at[name] = c.at[name].expand(T, many, *c.at[name].shape[2:]).contiguous()
    other.at["A"] = c.at["A"]
    if c.at["h_in"] is not None:
        other.at["h_in"] = c.at["h_in"].expand(many, H, K, V).contiguous()
    two = other.run(False)
    other.ctx.close()
    return one, {"y": two["y"][:, :1], "h_out": two["h_out"][:1]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,grow", [(800, 0.3125), (1600, 0.5), (2000, 1.25)])
@pytest.mark.parametrize("written", ["values", "strengths"])
def test_nothing_written(hts, dtype, T, grow, written):  # noqa: F811
    """Steps that lengthen by exp(grow), nothing written before the last 20 of them (no values, or strengths of 0): zeros until then, and what 20 steps make after.

    A step's roundings, of up to 64 x 64 + K terms of a column's size, are 8 sqrt(64 x 64 + K) u of it, as in `allowed`; here every later step lengthens them too, so they are added
    up with the steps' factors, from the first one that has something to round."""
    K, V, live = 16, 24, 20
    c = Case(hts, dtype, T, 1, 1, 1, K, V, softplus=False, state=False)
    grown(c, np.full(T, grow))
    name, none = ("v", 0.0) if written == "values" else ("b", -200.0)
    c.at[name][:T - live] = none
    c.wide[name] = host(c.at[name])
    if name == "b":
        c.wide[name][:T - live] = -1e5                 # a strength of nothing in binary64 too
    want, _ = c.oracle(False)
    one, two = alone_and_beside_others(hts, c, 100)
    step, off = 8 * np.sqrt(64 * 64 + K) * so.U, np.zeros((1, V))
    S = np.zeros((K, V))
    for t in range(T - live, T):                       # the definition again, with the roundings beside it
        k = c.wide["k"][t, 0, 0]
        k, al, be = k / np.sqrt((k * k).sum() + 1e-6), np.exp(c.wide["a"][t, 0, 0]), so.sigmoid(c.wide["b"][t, 0, 0])
        z = c.wide["v"][t, 0, 0] - al * (k @ S)
        S = al * S + be * k[:, None] * z
        off = al * off + step * (np.sqrt((S * S).sum(0)) + np.abs(c.wide["v"][t, 0, 0]))
        for got in (one, two):
            so.near(host(got["y"][t, 0]), want["y"][t, 0], c.more["scale"] * off / so.U, 1, HALF[dtype], f"y {t}")
    for got in (one, two):
        assert bool((got["y"][:T - live] == 0).all())
        so.near(host(got["h_out"][0, 0]), want["h_out"][0, 0], off / so.U * np.ones((K, 1)), 1, HALF["f32"], "h_out")
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,first,grow", [(1600, 1e-25, 0.3125), (1600, 1e17, -0.3125), (2400, 1e-12, 0.25), (1600, 1e25, -0.375)])
def test_there_and_back(hts, dtype, T, first, grow):  # noqa: F811
    """A state that is carried only (strengths of 0): 320 steps of exp(grow), 320 of its inverse, and so on, so that it ends where it began or 320 steps from there.  Every chunk
    rounds each entry for its factor, its split into parts and its sum, and each joint twice more: 8 for each of the chunks are plenty; the exponents are exact."""
    K, V = 24, 40
    c = Case(hts, dtype, T, 1, 1, 1, K, V, softplus=False)
    a = np.where(np.arange(T) // 320 % 2 == 0, grow, -grow)
    grown(c, a)
    c.at["b"][:] = -200.0
    c.at["h_in"] *= first
    one, two = alone_and_beside_others(hts, c, 100)
    want = host(c.at["h_in"]) * np.exp(a.sum())
    for got in (one, two):
        so.near(host(got["h_out"]), want, np.abs(want) * 8 * (T // 64 + 1), 1, HALF["f32"], "h_out")
        assert bool(got["y"].isfinite().all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_keys(hts, dtype):  # noqa: F811
    """Keys as they are, of a square of 6.25 at strengths of a half: each step turns the state along its key over and more than doubles it.  A state of nothing stays nothing."""
    T, K, V = 1600, 16, 24
    c = Case(hts, dtype, T, 1, 1, 1, K, V, softplus=False, normalize=False, state=False)
    grown(c, np.zeros(T))
    c.at["k"][:T - 10] = 0.625
    c.at["b"][:T - 10] = 0.0
    c.at["v"][:T - 10] = 0.0
    for name in ("k", "b", "v"):
        c.wide[name] = host(c.at[name])
    want, off = c.oracle(False)
    one, two = alone_and_beside_others(hts, c, 100)
    for got in (one, two):
        assert bool((got["y"][:T - 10] == 0).all())
        for name in ("y", "h_out"):
            so.near(host(got[name]), want[name], off[name] / so.U, 1, HALF[dtype if name == "y" else "f32"], name)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_episodes(hts, dtype):  # noqa: F811
    """A state that has left binary32 is not there for an episode that begins after it, in a segment of its own or in the middle of one."""
    T, K, V = 1600, 16, 24
    for begin in (640, 1000, 1599):
        c = Case(hts, dtype, T, 1, 1, 1, K, V, softplus=False, starts=0.5)
        s = np.zeros((T, 1), dtype=np.uint8)
        s[begin] = 1
        c.wide["starts"], c.at["starts"] = s, torch.from_numpy(s).cuda()
        a = np.where(np.arange(T) < begin, 0.5, -0.25)
        grown(c, a)
        got = c.run(False)
        y = host(got["y"])
        assert not np.isfinite(y[begin - 64]).any() and np.isfinite(y[begin:]).all() and bool(got["h_out"].isfinite().all())
        c.at["starts"][:] = 0
        c.at["starts"][begin] = 1
        c.at["h_in"] *= 0
        c.at["v"][:begin] = 0
        again = c.run(False)
        assert bool((again["y"][:begin] == 0).all()) and torch.equal(again["h_out"], got["h_out"]) and torch.equal(again["y"][begin:], got["y"][begin:])
        c.ctx.close()
