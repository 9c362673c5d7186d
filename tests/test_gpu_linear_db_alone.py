"""The bias' gradient alone, of inputs with fewer entries than a 16-byte word, over rows that are cut into slices: the values, and the bits that the call with
all gradients gives.  tests/test_linear_slices.py holds that the slices stay within the workspace."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from test_gpu_seq import HALF, TYPES, host, put

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["none", "silu"])
@pytest.mark.parametrize("M,N,K", [(513, 8, 1), (1024, 64, 1), (1500, 104, 3), (8192, 256, 2), (2100, 40, 7), (900, 33, 5), (1100, 64, 9)])
def test_db_alone(hts, dtype, kind, M, N, K):
    """db is a sum of M products of dy and a slope: a rounding for each addition, and 16 + 12 pre^2 of the slope's own (an exponent's grow with its square)."""
    r, ty = np.random.default_rng(M + N + K), TYPES[dtype]
    (x, _), (w, _), (pre, pre64), (dy, dy64) = (put(r.normal(size=s), ty) for s in ((M, K), (N, K), (M, N), (M, N)))
    act = getattr(hts, "ACT_" + kind.upper())
    ctx = hts.SeqContext(hts.linear_workspace(M, N, K, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32, act=act))
    db, whole, dw = torch.full((N,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda"), torch.empty(N, K, device="cuda")
    ctx.hts_linear_backward(x, w, dy, pre=pre if kind != "none" else None, act=act, db=db)
    ctx.hts_linear_backward(x, w, dy, pre=pre if kind != "none" else None, act=act, dw=dw, db=whole)
    torch.cuda.synchronize()
    want, size = (np.abs(dy64) * so.slope(pre64, kind, True) if s else dy64 * so.slope(pre64, kind) for s in (False, True))
    so.near(host(db), want.sum(0), size.sum(0), M + 8 + (0 if kind == "none" else 16 + 12 * np.abs(pre64).max() ** 2), HALF["f32"], "db")
    assert torch.equal(db, whole)
    ctx.close()
