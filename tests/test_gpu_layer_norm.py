"""Layer norm and its gradients against the definition in binary64 (delta_oracle.py), through the public entry points."""
import numpy as np
import pytest
import torch

import delta_oracle as do
import seq_oracle as so
from test_gpu_seq import HALF, TYPES, hts, host, inside, put, spread, untouched  # noqa: F401

pytestmark = pytest.mark.gpu

# one row and one entry; widths around a vector's, a wavefront's, and each of the kernels' limits; more rows than workgroups
SHAPES = [(1, 1), (1, 7), (3, 8), (16, 512), (5, 513), (7, 1023), (33, 1999), (3, 2048), (9, 2049), (2, 4097), (3, 8191), (2, 8200), (1, 16384), (2500, 96), (300, 4160)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", SHAPES)
@pytest.mark.parametrize("params,pad,shift", [(True, 0, 0), (False, 8, 8), (True, 3, 1)])
def test_layer_norm(hts, dtype, M, F, params, pad, shift):  # noqa: F811
    r, ty = np.random.default_rng(M + F), TYPES[dtype]
    (x, x64), (dy, dy64), (add, add64) = (put(r.normal(size=(M, F)) * (1 + r.random(F)) + o, ty) for o in (0.7, 0.0, 0.1))
    (w, w64), (b, b64) = (put(o + 0.2 * r.normal(size=F)) if params else (None, None) for o in (1.0, 0.0))
    use_add = pad != 8
    want, off = do.norm(x64, w64, b64, np.float64(np.float32(1e-5)), dy64, add64 if use_add else None)
    ctx = hts.SeqContext(hts.layer_norm_workspace(M, F, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32))
    wide_y, y = inside((M, F), ty, pad, shift)
    wide_dx, dx = inside((M, F), ty, pad, shift)
    dw, db = torch.full((F,), 7.0, device="cuda"), torch.full((F,), 7.0, device="cuda")
    xs = spread(x, pad, shift)
    ctx.hts_layer_norm(xs, y, w=w, b=b)
    args = dict(w=w, add=spread(add, pad, shift) if use_add else None)
    ctx.hts_layer_norm_backward(xs, spread(dy, pad, shift), dx=dx, dw=dw, db=db, **args)
    torch.cuda.synchronize()
    so.near(host(y), want["y"], off["y"] / so.U, 1, HALF[dtype], "y")
    so.near(host(dx), want["dx"], off["dx"] / so.U, 1, HALF[dtype], "dx")
    so.near(host(dw), want["dw"], off["dw"] / so.U, 1, HALF["f32"], "dw")
    so.near(host(db), want["db"], off["db"] / so.U, 1, HALF["f32"], "db")
    untouched(wide_y, F, shift)
    untouched(wide_dx, F, shift)
    # one output at a time, and in the place of what it comes from: the same bits
    for name, out in (("dx", dx), ("dw", dw), ("db", db)):
        alone = torch.empty_like(out).contiguous()
        ctx.hts_layer_norm_backward(x, dy, w=w, add=add if use_add else None, **{name: alone})
        assert torch.equal(alone, out), name
    for place in ("x", "dy") + (("add",) if use_add else ()):
        given = {"x": x.clone(), "dy": dy.clone(), "add": add.clone() if use_add else None}
        dw2 = torch.empty_like(dw)
        ctx.hts_layer_norm_backward(given["x"], given["dy"], w=w, add=given["add"], dx=given[place], dw=dw2)
        assert torch.equal(given[place], dx) and torch.equal(dw2, dw), place
    ctx.hts_layer_norm(x, x, w=w, b=b)
    assert torch.equal(x, y)
    ctx.close()


def test_rows_apart(hts):  # noqa: F811
    """Rows of one value, of what is not finite, beside others; one row for all."""
    ctx = hts.SeqContext(hts.layer_norm_workspace(6, 40))
    x = torch.randn(6, 40, device="cuda")
    x[1] = 3.5
    x[2, 7], x[4, 0] = float("nan"), float("inf")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    b = torch.randn(40, device="cuda")
    ctx.hts_layer_norm(x, y, b=b)
    dy = torch.randn(6, 40, device="cuda")
    dy[5, 3] = float("nan")
    ctx.hts_layer_norm_backward(x, dy, dx=dx)
    torch.cuda.synchronize()
    assert torch.equal(y[1], b) and bool(y[[2, 4]].isnan().all()) and bool(y[[0, 3, 5]].isfinite().all())
    assert bool(dx[[2, 4, 5]].isnan().all()) and bool(dx[[0, 1, 3]].isfinite().all())
    one = x[:1].expand(6, 40)
    ctx.hts_layer_norm(one, y, b=b)
    assert torch.equal(y[5], y[0]) and bool(y.isfinite().all())
    ctx.close()


def test_no_noise(hts):  # noqa: F811
    """A mean of a thousand deviations: what is left after it is taken off has its digits."""
    ctx = hts.SeqContext(0)
    r = np.random.default_rng(5)
    x, x64 = put(1000 + r.normal(size=(4, 777)))
    y = torch.empty_like(x)
    ctx.hts_layer_norm(x, y, eps=0.0)
    want, off = do.norm(x64, None, None, 0.0)
    so.near(host(y), want["y"], off["y"] / so.U, 1, HALF["f32"], "y")
    ctx.close()


@pytest.mark.parametrize("M,F", [(3, 100), (9, 1500), (1, 6000)])
def test_no_eps(hts, M, F):  # noqa: F811
    """Rows that are not there have no deviations, and without eps no inverse of them: nothing of it reaches the sums."""
    ctx = hts.SeqContext(hts.layer_norm_workspace(M, F))
    r = np.random.default_rng(6)
    (x, x64), (dy, dy64) = put(r.normal(size=(M, F))), put(r.normal(size=(M, F)))
    dx, dw, db = torch.empty_like(x), torch.empty(F, device="cuda"), torch.empty(F, device="cuda")
    ctx.hts_layer_norm_backward(x, dy, dx=dx, dw=dw, db=db, eps=0.0)
    want, off = do.norm(x64, None, None, 0.0, dy64)
    for name, got in (("dx", dx), ("dw", dw), ("db", db)):
        so.near(host(got), want[name], off[name] / so.U, 1, HALF["f32"], name)
    ctx.close()
