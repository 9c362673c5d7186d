"""The gated delta rule's gates where they are at their limits."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from test_gpu_delta_rule import Case
from test_gpu_seq import HALF, hts, host, put  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 16, 17, 130])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), -1e4, 1e38])
def test_a_first_step_has_no_decay(hts, dtype, T, value):  # noqa: F811
    """alpha is 0 where a step begins an episode, whatever its input: of calls of a few steps as of long ones, of outputs as of gradients."""
    c = Case(hts, dtype, T, 2, 1, 2, 16, 40, starts=0.5, softplus=False)
    s = np.zeros((T, 2), dtype=np.uint8)
    for t in {0, T // 2, T - 1}:
        s[t, 0] = 1
        c.at["a"][t, 0] = value                        # (A is -1: a growth that no number holds, or a step that forgets)
        c.wide["a"][t, 0] = 0.0                        # the oracle's factor is 0 there, and times infinity no number
    c.wide["starts"], c.at["starts"] = s, torch.from_numpy(s).cuda()
    got = c.run()
    want, off = c.oracle()
    for name in got:
        so.near(host(got[name]), want[name], off[name] / so.U, 1, HALF["f32" if got[name].dtype is torch.float32 else dtype], name)
    assert bool((got["da"][torch.from_numpy(s).cuda() != 0] == 0).all())
    c.ctx.close()


@pytest.mark.parametrize("T", [12, 130])
@pytest.mark.parametrize("name,value", [("a", float("nan")), ("a", -1e4), ("b", float("nan"))])
def test_gradients_before_a_gate_that_is_no_number(hts, T, name, value):  # noqa: F811
    """A decay that is no number is a factor of the state's gradient on its way to the steps before it, and to the state that the sequence began with; a strength is one of what a
    step takes away.  The episode before has nothing of it."""
    c = Case(hts, "f32", T, 2, 1, 2, 16, 40, starts=0.5, softplus=False)
    s = np.zeros((T, 2), dtype=np.uint8)
    s[T // 4, 1] = 1                                  # the second sequence: an episode begins a quarter into it
    c.wide["starts"], c.at["starts"] = s, torch.from_numpy(s).cuda()
    at = T // 2
    c.at[name][at] = value
    got = c.run()
    for n, first in ((0, 0), (1, T // 4)):
        for g in ("dk", "dv"):
            assert bool(got[g][first:at + 1, n].isnan().all()), (g, n)
        assert bool(got["y"][at:, n].isnan().all()) and bool(got["h_out"][n].isnan().all()) and bool(got["y"][:at, n].isfinite().all())
    for g in ("dq", "dk", "dv", "da", "db"):
        assert bool(got[g][:T // 4, 1].isfinite().all()), g
    assert bool(got["dh_in"][0].isnan().all()) and bool(got["dh_in"][1].isfinite().all())
    c.ctx.close()


@pytest.mark.parametrize("T", [5, 90])
def test_strengths_next_to_one(hts, T):  # noqa: F811
    """db has a factor 1 - beta, which has digits where beta has none left of them.  The logistic function's own roundings: |b| for the product with log2(e), |b| for that number and
    eight more, on what the products of the two columns are off by."""
    c = Case(hts, "f32", T, 1, 1, 2, 16, 16)
    b = np.linspace(-20.0, 40.0, 2 * T).reshape(T, 1, 2)
    c.at["b"], c.wide["b"] = put(b)
    got = c.run()
    want, off = c.oracle()
    rest, share = so.sigmoid(-c.wide["b"]), so.sigmoid(c.wide["b"])
    # the oracle's db has 1 - beta as a difference, which is nothing in binary64 either from b = 37 on: from its dv = beta dz / d(beta z), and z step by step
    S, unit = c.wide["h_in"][0].copy(), lambda x: x / np.sqrt((x * x).sum() + 1e-6)
    for t in range(T):
        k = unit(c.wide["k"][t, 0, 0])
        al = np.exp(np.logaddexp(0, c.wide["a"][t, 0] + c.wide["a_bias"]) * c.wide["A"])[:, None, None]
        z = c.wide["v"][t, 0] - (k[:, None] * al * S).sum(1)
        S = al * S + share[t, 0][:, None, None] * k[:, None] * z[:, None]
        want["db"][t, 0] = (want["dv"][t, 0] * z).sum(1) * rest[t, 0]
    room = off["db"] / so.U * rest * share + np.abs(want["db"]) * (2 * np.abs(c.wide["b"]) + 8)
    so.near(host(got["db"]), want["db"], room, 1, HALF["f32"], "db")
    assert bool((got["db"] != 0).all())
    c.ctx.close()
