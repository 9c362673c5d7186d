"""Layer norm of rows whose squares are beyond binary32, or below it: the rule's values are ordinary numbers."""
import numpy as np
import pytest
import torch

import delta_oracle as do
import seq_oracle as so
from test_gpu_seq import HALF, TYPES, hts, host, put  # noqa: F401

pytestmark = pytest.mark.gpu


# each of the kernels' widths, rows beside one another in a workgroup that are large and that are not, and more rows than the largest grids have at a time
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", [(9, 100), (5, 700), (7, 1500), (4, 3000), (3, 6000), (3, 9001), (9001, 72), (2601, 1100), (600, 4200)])
@pytest.mark.parametrize("size,eps", [(1e20, 1e-5), (1e30, 1e-5), (3e37, 0.0), (1e-22, 0.0), (1e-30, 0.0), (1e-25, 1e-36), (4e-38, 0.0), (1e-40, 0.0)])
def test_rows_of_any_size(hts, dtype, M, F, size, eps):  # noqa: F811
    """Every second row is of that size, the others of one: those come out as they do alone.  Tolerances as for rows of ordinary numbers, which a power of two makes of each; gradients of
    small rows are as large as their sizes' inverses, and are compared where binary32 has them."""
    r, ty = np.random.default_rng(M + F), TYPES[dtype]
    scale = np.where(np.arange(M) % 2 == 0, size, 1.0)[:, None]
    (x, x64), (dy, dy64) = put((r.normal(size=(M, F)) * (1 + r.random(F)) + 0.3) * scale, ty), put(r.normal(size=(M, F)) * np.minimum(scale, 1.0), ty)
    (w, w64), (b, b64) = (put(o + 0.2 * r.normal(size=F)) for o in (1.0, 0.0))
    if size < 1e-39 and dtype == "bf16":               # (a few of the type's smallest numbers)
        x[::2] = x[::2].abs()
        x64 = host(x)
    want, off = do.norm(x64, w64, b64, float(np.float32(eps)), dy64)
    # Gradients of the smallest numbers are such numbers, whose products are rounded to multiples of 2^-149, not relative to themselves: g = dy w once, mean(g) by its terms (on average) and its
    # division, mean(g h) by its additions (half a step each, over F of them), its terms and its division, times h, and the last difference: (4 + 3 |h|) half steps, which r makes of a size
    # (nothing for rows of one)
    d = x64 - x64.mean(1, keepdims=True)
    s = np.sqrt((d * d).mean(1, keepdims=True) + float(np.float32(eps)))
    off["dx"] = off["dx"] + (4 + 3 * np.abs(d / s)) * 2.0 ** -150 / s
    ctx = hts.SeqContext(hts.layer_norm_workspace(M, F, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32))
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(F, device="cuda"), torch.empty(F, device="cuda")
    ctx.hts_layer_norm(x, y, w=w, b=b, eps=eps)
    ctx.hts_layer_norm_backward(x, dy, w=w, dx=dx, dw=dw, db=db, eps=eps)
    torch.cuda.synchronize()
    so.near(host(y), want["y"], off["y"] / so.U, 1, HALF[dtype], "y")
    so.near(host(dx), want["dx"], off["dx"] / so.U, 1, HALF[dtype], "dx")          # (large rows' are 1e-37 or less: any such number is within that)
    so.near(host(dw), want["dw"], off["dw"] / so.U, 1, HALF["f32"], "dw")
    so.near(host(db), want["db"], off["db"] / so.U, 1, HALF["f32"], "db")
    # in the place of what it comes from: the same bits
    for place in (x.clone(), dy.clone()):
        given = (place, dy) if torch.equal(place, x) else (x, place)
        ctx.hts_layer_norm_backward(*given, w=w, dx=place, dw=torch.empty_like(dw), eps=eps)
        assert torch.equal(place, dx)
    ordinary = [torch.empty_like(x) for _ in range(2)]
    x[::2], dy[::2] = 1.0, 0.0
    x[::2, 0] = 2.0
    ctx.hts_layer_norm(x, ordinary[0], w=w, b=b, eps=eps)
    ctx.hts_layer_norm_backward(x, dy, w=w, dx=ordinary[1], eps=eps)
    assert torch.equal(ordinary[0][1::2], y[1::2]) and torch.equal(ordinary[1][1::2], dx[1::2])
    ctx.close()


@pytest.mark.parametrize("F", [100, 1500, 9001])
def test_what_is_not_finite_stays(hts, F):  # noqa: F811
    """Infinities and NaN make their row NaN, whatever the other entries' size; rows of zeros without eps are NaN (0 / 0), with it they are the bias."""
    ctx = hts.SeqContext(0)
    x, b = torch.randn(6, F, device="cuda"), torch.randn(F, device="cuda")
    x[0], x[1], x[2] = x[0] * 1e30, x[1] * 1e-30, 0
    x[0, 1], x[1, 2], x[3, 0] = float("nan"), float("inf"), -float("inf")
    y = torch.empty_like(x)
    ctx.hts_layer_norm(x, y, b=b)
    assert bool(y[[0, 1, 3]].isnan().all()) and torch.equal(y[2], b) and bool(y[4:].isfinite().all())
    ctx.hts_layer_norm(x, y, b=b, eps=0.0)
    assert bool(y[[0, 1, 2, 3]].isnan().all()) and bool(y[4:].isfinite().all())
    ctx.close()
