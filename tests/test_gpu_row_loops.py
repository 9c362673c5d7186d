"""Layer norm and AdamW where a workgroup goes round: more rows, and more pieces of a plan, than the largest grid has at a time."""
import numpy as np
import pytest
import torch

import delta_oracle as do
import seq_oracle as so
from seq_oracle import U
from test_gpu_seq import HALF, TYPES, hts, host, put  # noqa: F401

pytestmark = pytest.mark.gpu

# (the grids of 256 units take 4096 rows of up to 1024 entries, 1024 of up to 4096, 512 above, and backward 4096, 1024 and 256)
SHAPES = [(9001, 96), (4099, 520), (2500, 1500), (1500, 2600), (1301, 4160), (600, 9000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F", SHAPES)
@pytest.mark.parametrize("use_add", [True, False])
def test_more_rows_than_workgroups(hts, dtype, M, F, use_add):  # noqa: F811
    r, ty = np.random.default_rng(M + F), TYPES[dtype]
    (x, x64), (dy, dy64), (add, add64) = (put(r.normal(size=(M, F)) * (1 + r.random(F)) + o, ty) for o in (0.7, 0.0, 0.1))
    (w, w64), (b, b64) = (put(o + 0.2 * r.normal(size=F)) for o in (1.0, 0.0))
    add, add64 = (add, add64) if use_add else (None, None)
    want, off = do.norm(x64, w64, b64, np.float64(np.float32(1e-5)), dy64, add64)
    ctx = hts.SeqContext(hts.layer_norm_workspace(M, F, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32))
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(F, device="cuda"), torch.empty(F, device="cuda")
    ctx.hts_layer_norm(x, y, w=w, b=b)
    ctx.hts_layer_norm_backward(x, dy, w=w, add=add, dx=dx, dw=dw, db=db)
    torch.cuda.synchronize()
    for name, got in (("y", y), ("dx", dx), ("dw", dw), ("db", db)):
        so.near(host(got), want[name], off[name] / so.U, 1, HALF["f32" if got.dtype is torch.float32 else dtype], name)
    # in the place of what it comes from, with the next row on its way: the same bits
    for place in ("x", "dy") + (("add",) if use_add else ()):
        given = {"x": x.clone(), "dy": dy.clone(), "add": add.clone() if use_add else None}
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        ctx.hts_layer_norm_backward(given["x"], given["dy"], w=w, add=given["add"], dx=given[place], dw=dw2, db=db2)
        assert torch.equal(given[place], dx) and torch.equal(dw2, dw) and torch.equal(db2, db), place
    ctx.hts_layer_norm(x, x, w=w, b=b)
    assert torch.equal(x, y)
    ctx.close()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("sizes", [[2048 * 1023 + 5], [2048 * 1024 + 1, 3, 2048 * 1500 + 77, 5000]])
def test_more_pieces_than_workgroups(hts, half, sizes):  # noqa: F811
    """The gradients' norm over more pieces than a workgroup has at a time, and more than two: by entries of one place each, and over all of them.  The norm is a root of a sum in
    64 bits, rounded once."""
    r = np.random.default_rng(len(sizes))
    z = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    tensors = []
    for n in sizes:
        g = torch.from_numpy(r.normal(size=n) * np.exp(r.normal(size=n))).to(torch.bfloat16 if half else torch.float32).cuda()
        tensors.append(hts.AdamWTensor(z(n), g, z(n), z(n)))
    opt, hp, norm = hts.AdamW(tensors), hts.AdamWHParams(lr=1e-3, max_grad_norm=0.5), z(1)
    size = np.sqrt(sum((host(t.g) ** 2).sum() for t in tensors))
    opt.hts_adamw_step(hp, grad_norm=norm)
    torch.cuda.synchronize()
    assert abs(float(norm) - size) <= 2 * U * size
    for t in tensors:                                  # the first moment of a beginning: (1 - beta1) g clipped; 8 roundings as in the tests of a step
        want = host(t.g) * min(1.0, 0.5 / (size + 1e-6)) * (1 - float(np.float32(hp.beta1)))
        assert (np.abs(host(t.m) - want) <= 9 * U * np.abs(want)).all()
    # one entry alone, wherever it lies
    total = np.cumsum([0, *sizes])
    for at in (0, 2047, 2048 * 1023 - 1, 2048 * 1023, 2048 * 1024, int(total[-1]) - 1, 2048 * 2048 + 9):
        if at >= total[-1]:
            continue
        i = int(np.searchsorted(total, at, side="right")) - 1
        for t in tensors:
            t.g.zero_()
        tensors[i].g[at - int(total[i])] = -3.0
        opt.hts_adamw_step(hp, grad_norm=norm)
        torch.cuda.synchronize()
        assert float(norm) == 3.0, at
    opt.close()
