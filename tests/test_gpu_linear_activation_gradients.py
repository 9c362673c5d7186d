"""bfloat16 gradients through an activation: g = dy act'(pre), which has 24 bits, reaches dx, dw and db as three bfloat16 numbers, so that nothing of it is lost that counts
in binary32.  Tolerances: half a step of the output's type, and binary32 roundings of the sum of its terms' sizes: two for each of a term's three products and additions,
eight for the rest, and the slope's own (16 + 12 pre^2, since an exponent's grow with its square)."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from test_gpu_seq import HALF, host, put

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def context(hts, M, N, K, act):
    return hts.SeqContext(hts.linear_workspace(M, N, K, precision=hts.PRECISION_BF16, act=act))


@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("M,N,K,pad,shift", [(1, 512, 512, 0, 0), (33, 64, 129, 8, 8), (80, 531, 517, 3, 1), (5, 3, 2000, 0, 0), (700, 40, 33, 0, 0), (384, 640, 256, 16, 0), (1030, 136, 200, 0, 0), (2, 8, 8, 0, 0)])
def test_dx(hts, kind, M, N, K, pad, shift):
    r = np.random.default_rng(M + 3 * N + K)
    (w, w64), (pre, pre64), (dy, dy64), (x, _), (add, add64) = (put(r.normal(size=s), torch.bfloat16) for s in ((N, K), (M, N), (M, N), (M, K), (M, K)))
    act = getattr(hts, "ACT_" + kind.upper())
    ctx = context(hts, M, N, K, act)
    wide = torch.zeros(M, K + pad + shift, dtype=torch.bfloat16, device="cuda")
    dx = wide[:, shift:shift + K]
    use_add = kind != "relu"
    ctx.hts_linear_backward(x, w, dy, pre=pre, act=act, add=add if use_add else None, dx=dx)
    torch.cuda.synchronize()
    want, size = (so.linear_grad(np.zeros((M, K)), w64, pre64, dy64, add64 if use_add else None, kind, size=s)[0] for s in (False, True))
    so.near(host(dx), want, size, 6 * N + 8 + 16 + 12 * np.abs(pre64).max() ** 2, HALF["bf16"], "dx")
    ctx.close()


@pytest.mark.parametrize("M", [1, 700])
def test_three_numbers_and_no_fewer(hts, M):
    """dw and db of a gradient that needs all of its 24 bits: one row that counts, so that db is g and dw g times x with nothing added.  Two numbers (16 bits and a sign) leave
    2^-18 of it, three nothing: allowed are 4 roundings of 2^-24 against the slope in binary32 as the same formula gives it in any order, which its own 16 + 12 pre^2 roundings
    blur; the pre-activations are small, so that these are 16 to 19, half of what a third number is worth (2^-18 is 64 of them)."""
    N, K = 64, 64
    r = np.random.default_rng(M)
    pre, pre64 = put(r.uniform(-0.5, 0.5, size=(M, N)), torch.bfloat16)
    dy64 = np.zeros((M, N))
    dy64[M // 2] = r.uniform(0.5, 1.0, size=N) * r.choice((-1, 1), size=N)
    dy, dy64 = put(dy64, torch.bfloat16)
    x, x64 = put(r.uniform(0.5, 1.0, size=(M, K)), torch.bfloat16)
    w, _ = put(r.normal(size=(N, K)), torch.bfloat16)
    ctx = context(hts, M, N, K, hts.ACT_SILU)
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ctx.hts_linear_backward(x, w, dy, pre=pre, act=hts.ACT_SILU, dw=dw, db=db)
    torch.cuda.synchronize()
    g = (dy64 * so.slope(pre64, "silu"))[M // 2]
    # some gradient has to be further than that from what two numbers hold, or this would say nothing
    first = torch.from_numpy(g).float().bfloat16().double().numpy()
    two = first + torch.from_numpy(g - first).float().bfloat16().double().numpy()
    assert (np.abs(g - two) > 40 * so.U * np.abs(g)).any()
    so.near(host(db), g, np.abs(g), 4 + 16 + 12 * 0.25, 0, "db")
    so.near(host(dw), g[:, None] * x64[M // 2], np.abs(g[:, None] * x64[M // 2]), 4 + 16 + 12 * 0.25, 0, "dw")
    ctx.close()


def test_a_gradient_beyond_bfloat16(hts):
    """dy is bfloat16's largest number and the slope a little over 1: g is within binary32 and beyond bfloat16, which would round it to infinity."""
    largest = float(torch.finfo(torch.bfloat16).max)
    pre64 = np.array([[p for p in np.arange(0.5, 3, 1 / 128) if 1.0020 < so.slope(np.array(p), "silu") < 1.0038]])
    N, K = pre64.shape[1], 8
    assert N > 0
    pre, dy = torch.from_numpy(pre64).bfloat16().cuda(), torch.full((1, N), largest, dtype=torch.bfloat16, device="cuda")
    dy[0, ::2] = -largest
    x, w = (torch.full(s, 2.0 ** -100, dtype=torch.bfloat16, device="cuda") for s in ((1, K), (N, K)))
    ctx = context(hts, 1, N, K, hts.ACT_SILU)
    dx, dw, db = torch.empty(1, K, dtype=torch.bfloat16, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ctx.hts_linear_backward(x, w, dy, pre=pre, act=hts.ACT_SILU, dx=dx, dw=dw, db=db)
    torch.cuda.synchronize()
    g = host(dy)[0] * so.slope(host(pre)[0], "silu")
    assert bool((np.abs(g) > largest).all())
    so.near(host(db), g, np.abs(g), 4 + 16 + 12 * 2.25, 0, "db")
    so.near(host(dw), g[:, None] * host(x), np.abs(g[:, None] * host(x)), 4 + 16 + 12 * 2.25, 0, "dw")
    so.near(host(dx), g[None] @ host(w), np.abs(g)[None] @ host(w), 6 * N + 24 + 12 * 2.25, HALF["bf16"], "dx")
    ctx.close()
