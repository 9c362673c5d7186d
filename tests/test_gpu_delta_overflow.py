"""The gated delta rule where a state leaves binary32 on its way through a chunk: by values, by keys that lengthen it, by decays above one.  Other episodes (before it, after it, in
the same chunk), other sequences and other columns of values have nothing of it, in outputs, states and gradients."""
import numpy as np
import pytest
import torch

from test_gpu_delta_rule import Case
from test_gpu_seq import hts, host  # noqa: F401

pytestmark = pytest.mark.gpu


def spoil(c, how, first, last):
    """Steps first .. last of the first sequence, of every head."""
    if how == "values":                                       # of one column
        c.at["k"][first:last, 0] = c.at["k"][first, 0].clone()
        c.at["b"][first:last, 0] = 30.0
        sign = torch.where(torch.arange(last - first, device="cuda") % 2 == 0, 3e38, -3e38)
        c.at["v"][first:last, 0, :, 3] = sign[:, None].to(c.ty)
    elif how == "keys":
        c.at["k"][first:last, 0] = 60.0
        c.at["b"][first:last, 0] = 30.0
    else:                                                     # "decays" (A is -1)
        c.at["a"][first:last, 0] = -20.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["values", "keys", "decays"])
@pytest.mark.parametrize("T,first,last", [(130, 20, 44), (130, 70, 100), (130, 33, 64), (64, 0, 40), (200, 100, 190), (900, 400, 440)])
def test_other_episodes(hts, dtype, how, T, first, last):  # noqa: F811
    N, G, H, K, V = 2, 1, 2, 16, 40
    if T == 900:
        N = 1
    make = lambda: Case(hts, dtype, T, N, G, H, K, V, starts=0.5, softplus=False, normalize=how != "keys")  # noqa: E731
    base, c = make(), make()
    s = np.zeros((T, N), dtype=np.uint8)
    s[[first, last], 0] = 1
    for x in (base, c):
        x.at["starts"] = torch.from_numpy(s).cuda()
        x.at["dy"][first:last, 0] = 0                          # what reaches the spoilt episode's gradients from its own outputs is nothing
    spoil(c, how, first, last)
    want, got = base.run(), c.run()
    off = 1e-5 if dtype == "f32" else 2.0 ** -7
    near = lambda a, b: bool(np.isfinite(host(a)).all()) and np.allclose(host(a), host(b), rtol=off, atol=off * float(b.float().abs().max()))  # noqa: E731
    assert not bool(got["y"][first:last, 0].isfinite().all())
    for name in ("y", "dq", "dk", "dv", "da", "db"):
        assert near(got[name][:first, 0], want[name][:first, 0]) if first else True, name
        assert near(got[name][last:, 0], want[name][last:, 0]), name
        if N > 1:
            assert near(got[name][:, 1], want[name][:, 1]), name
    if how == "values":
        keep = [v for v in range(V) if v != 3]
        assert bool(got["y"][:, :, :, keep].isfinite().all()) and bool(got["y"][first, 0].isfinite().all())
    assert near(got["h_out"], want["h_out"]) and (first == 0 or near(got["dh_in"], want["dh_in"]))
    base.ctx.close()
    c.ctx.close()
