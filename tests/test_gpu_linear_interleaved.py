"""Operands and outputs that lie between each other's rows in one wider array share nothing and are taken: the values that separate arrays give."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 40, 24), (70, 72, 40), (300, 33, 65)])
def test_parts_of_one_array(hts, dtype, M, N, K):
    prec = hts.PRECISION_BF16 if dtype is torch.bfloat16 else hts.PRECISION_FP32
    x, w, res = torch.randn(M, K, device="cuda").to(dtype), torch.randn(N, K, device="cuda").to(dtype), torch.randn(M, N, device="cuda").to(dtype)
    ctx = hts.SeqContext(hts.linear_workspace(M, N, K, precision=prec, act=hts.ACT_SILU))
    y, pre, dx, dw, db = torch.empty_like(res), torch.empty_like(res), torch.empty_like(x), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ctx.hts_linear(x, w, y, residual=res, pre=pre, act=hts.ACT_SILU)
    ctx.hts_linear_backward(x, w, res, pre=pre, act=hts.ACT_SILU, add=x, dx=dx, dw=dw, db=db)
    wide = torch.zeros(M, 2 * K + 3 * N, dtype=dtype, device="cuda")
    xs, dxs, ys, rs, ps = wide[:, :K], wide[:, K:2 * K], wide[:, 2 * K:2 * K + N], wide[:, 2 * K + N:2 * K + 2 * N], wide[:, 2 * K + 2 * N:]
    xs.copy_(x)
    rs.copy_(res)
    dws, dbs = torch.empty_like(dw), torch.empty_like(db)
    ctx.hts_linear(xs, w, ys, residual=rs, pre=ps, act=hts.ACT_SILU)
    ctx.hts_linear_backward(xs, w, rs, pre=ps, act=hts.ACT_SILU, add=xs, dx=dxs, dw=dws, db=dbs)
    torch.cuda.synchronize()
    for a, b in ((ys, y), (ps, pre), (dxs, dx), (dws, dw), (dbs, db), (xs, x), (rs, res)):
        assert torch.equal(a, b)
    with pytest.raises(hts.HtsError):
        ctx.hts_linear(xs, w, wide[:, K - 1:K - 1 + N], residual=rs)
    with pytest.raises(hts.HtsError):
        ctx.hts_linear_backward(xs, w, rs, dx=wide[:, 2 * K + N - 1:3 * K + N - 1], dw=dws)
    ctx.close()
