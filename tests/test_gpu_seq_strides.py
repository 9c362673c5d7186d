"""Rows and steps of the sequence memory's operands at unusual distances: one row for all, rows that overlap, a single row or step whose distance says
nothing.  Values against the definitions in binary64 (seq_oracle.py), with the tolerances of test_gpu_seq.py."""
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
@pytest.mark.parametrize("M,N,K", [(100, 64, 72), (33, 16, 8), (700, 128, 40)])
@pytest.mark.parametrize("step", [0, 8])
def test_gradients_of_rows_that_overlap(hts, dtype, M, N, K, step):
    """dy and x as one row for all (step 0) or as windows of a longer row, 8 entries apart: the reduction over the rows ends with the last one."""
    r, ty = np.random.default_rng(M + step), TYPES[dtype]
    (x, x64), (w, w64), (dy, dy64) = put(r.normal(size=(step * (M - 1) + K)), ty), put(r.normal(size=(N, K)), ty), put(r.normal(size=(step * (M - 1) + N)), ty)
    window = lambda a, cols: a.as_strided((M, cols), (step, 1)) if torch.is_tensor(a) else np.stack([a[step * m:step * m + cols] for m in range(M)])  # noqa: E731
    ctx = hts.SeqContext(hts.linear_workspace(M, N, K, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32))
    dx, dw, db = torch.empty(M, K, dtype=ty, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ctx.hts_linear_backward(window(x, K), w, window(dy, N), dx=dx, dw=dw, db=db)
    torch.cuda.synchronize()
    want, size = (so.linear_grad(window(x64, K), w64, None, window(dy64, N), None, "none", size=s) for s in (False, True))
    so.near(host(dx), want[0], size[0], 2 * N + 8, HALF[dtype], "dx")
    so.near(host(dw), want[1], size[1], 2 * M + 8, HALF["f32"], "dw")
    so.near(host(db), want[2], size[2], M + 8, HALF["f32"], "db")
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_single_row_or_step_has_no_distance(hts, dtype):
    """Views of one row, step or sequence whose strides lead far beyond their array give what plain ones do."""
    ty = TYPES[dtype]
    far = (1 << 24) + 24
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g).to(ty)  # noqa: E731
    loose = lambda t, *st: t.as_strided(t.shape, (*st, *t.stride()[len(st):]))  # noqa: E731
    prec = hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32
    ctx = hts.SeqContext(max(hts.linear_workspace(1, 40, 64, precision=prec), hts.short_conv_workspace(7, 3, 48, 4, precision=prec), hts.selective_scan_workspace(7, 3, 48, 16, precision=prec)))
    x, w = normal(1, 64), normal(40, 64)
    out = [torch.empty(1, 40, dtype=ty, device="cuda") for _ in range(2)]
    ctx.hts_linear(x, w, out[0])
    ctx.hts_linear(loose(x, far * far), w, loose(out[1], 1))
    assert torch.equal(*out)
    for T, N in ((1, 3), (7, 1)):
        D, S, W = 48, 16, 4
        loosen = lambda t: loose(t, far * far) if T == 1 else loose(t, t.stride(0), far * far)  # noqa: E731
        taps = torch.randn(D, W, device="cuda", generator=g)
        x, dt, z, B, C, dy = (normal(T, N, k) for k in (D, D, D, S, S, D))
        A, state, h = -torch.rand(D, S, device="cuda", generator=g), torch.randn(N, W - 1, D, device="cuda", generator=g), torch.randn(N, D, S, device="cuda", generator=g)
        results = []
        for way in (lambda t: t, loosen):
            y, dx, dw, v, held, saw = (torch.empty(*s, dtype=ty, device="cuda") if s[0] == T else torch.empty(*s, device="cuda") for s in ((T, N, D), (T, N, D), (D, W), (T, N, D), (N, D, S), (N, W - 1, D)))
            ctx.hts_short_conv(way(x), taps, way(y), act=hts.ACT_SILU, state_in=state, state_out=saw)
            ctx.hts_short_conv_backward(way(x), taps, way(dy), way(dx), dw, act=hts.ACT_SILU, state_in=state)
            states = torch.empty(hts.selective_scan_states(T, N, D, S), device="cuda")
            ctx.hts_selective_scan(way(x), way(dt), A, way(B), way(C), way(v), z=way(z), h_in=h, h_out=held, states=states)
            grads = [torch.empty_like(t) for t in (x, dt, B, C, z)]
            dA = torch.empty_like(A)
            ctx.hts_selective_scan_backward(way(x), way(dt), A, way(B), way(C), way(dy), states, way(grads[0]), way(grads[1]), way(grads[2]), way(grads[3]), dA, z=way(z), dz=way(grads[4]), h_in=h)
            torch.cuda.synchronize()
            results.append([y, dx, dw, v, held, saw, dA, *grads])
        for a, b in zip(*results):
            assert torch.equal(a, b)
    ctx.close()
