"""Operands whose rows, steps and sequences lie so far apart that their offsets pass 31 and 32 bits, and contexts on a range of compute units.  The same bits as from compact
operands where the kernels are the same ones; on fewer units there are fewer segments, so values there are held against binary64 with the tolerances of test_gpu_seq.py."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from test_gpu_seq import HALF, WAYS, forward, scan_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def apart(whole, first, t, *strides):
    """t's values in `whole`, from entry `first` on, at those distances."""
    view = whole.as_strided(t.shape, (*strides, *t.stride()[len(strides):]), first)
    view.copy_(t)
    return view


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("word", [0, 1])                       # rows that are whole 16-byte words, and others
def test_rows_far_apart(hts, dtype, word):
    """Every operand of the products with rows 8 MB apart, 5.9 GB in all: as rows of C, as what the reduction goes along and as what it goes across."""
    size = torch.finfo(dtype).bits // 8
    far, M, N, K = (8 << 20) // size - (64 + word), 700, 72, 64
    whole = torch.zeros(M * far + 1024, dtype=dtype, device="cuda")
    prec = hts.PRECISION_BF16 if dtype is torch.bfloat16 else hts.PRECISION_FP32
    ctx = hts.SeqContext(max(hts.linear_workspace(*s, precision=prec, act=hts.ACT_SILU) for s in ((M, N, K), (N, M, K))))
    normal = lambda *s: torch.randn(*s, device="cuda").to(dtype)  # noqa: E731
    for rows, outputs in ((M, N), (N, M)):                     # x and the outputs far apart, then w too
        x, w, dy = normal(rows, K), normal(outputs, K), normal(rows, outputs)
        compact = [torch.empty(rows, outputs, dtype=dtype, device="cuda") for _ in range(2)] + [torch.empty(rows, K, dtype=dtype, device="cuda")]
        dw, db = torch.empty(outputs, K, device="cuda"), torch.empty(outputs, device="cuda")
        # the same rows' distances modulo 16 bytes, so that the same kernels run
        wide = lambda t: apart(torch.zeros(t.shape[0] * (t.shape[1] + 16 + word), dtype=dtype, device="cuda"), 0, t, (t.shape[1] + 16) // 8 * 8 + word)  # noqa: E731
        cx, cw, cg = wide(x), wide(w), wide(dy)
        ctx.hts_linear(cx, cw, compact[0], pre=compact[1], act=hts.ACT_SILU)
        ctx.hts_linear_backward(cx, cw, cg, pre=compact[1], act=hts.ACT_SILU, dx=compact[2], dw=dw, db=db)
        fx, fw, fg = apart(whole, 0, x, far), apart(whole, 128, w, far), apart(whole, 256, dy, far) if outputs == N else cg
        y, pre = (whole.as_strided((rows, outputs), (far, 1), 512 + 128 * i) if outputs == N else torch.empty_like(compact[i]) for i in range(2))
        dx, fdw, fdb = whole.as_strided((rows, K), (far, 1), 768), torch.empty_like(dw), torch.empty_like(db)
        ctx.hts_linear(fx, fw, y, pre=pre, act=hts.ACT_SILU)
        ctx.hts_linear_backward(fx, fw, fg, pre=pre, act=hts.ACT_SILU, dx=dx, dw=fdw, db=fdb)
        torch.cuda.synchronize()
        for name, a, b in zip(("y", "pre", "dx", "dw", "db"), (y, pre, dx, fdw, fdb), (*compact, dw, db)):
            assert torch.equal(a, b), (rows, outputs, name)
    ctx.close()


@pytest.mark.parametrize("T,N,st,sn", [(300, 1, 1 << 24, 0), (40, 3, 2048, (1 << 31) + 64), (40, 3, 2049, (1 << 31) + 67)])
def test_steps_and_sequences_far_apart(hts, T, N, st, sn):
    """All operands of the convolution and the scan, and their outputs, in one array of 10 or 13 GB."""
    dtype, D, S, W = torch.bfloat16, 64, 16, 4
    whole = torch.zeros(max(T * st, (N - 1) * sn + T * st) + 4096, dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(T)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, dt, z, dy = (normal(T, N, D).to(dtype) for _ in range(4))
    B, C = (normal(T, N, S).to(dtype) for _ in range(2))
    A, skip, bias, h, taps, state = -torch.exp(normal(D, S)), normal(D), normal(D) - 2, normal(N, D, S), normal(D, W), normal(N, W - 1, D)
    ctx = hts.SeqContext(max(hts.short_conv_workspace(T, N, D, W, precision=hts.PRECISION_BF16), hts.selective_scan_workspace(T, N, D, S, precision=hts.PRECISION_BF16)))
    odd, results = st % 2, []
    for far in (False, True):
        places = iter(range(0, 2048, 80))
        if far:
            put = lambda t: apart(whole, next(places), t, st, sn)  # noqa: E731
        else:                                                  # distances that are multiples of the same
            put = lambda t: apart(torch.zeros(T * N * 112 + 112, dtype=dtype, device="cuda"), 0, t, N * (96 + odd), 96 + odd)  # noqa: E731
        new = lambda k: put(torch.zeros(T, N, k, dtype=dtype, device="cuda"))  # noqa: E731
        fx, fdt, fz, fdy, fB, fC = (put(t) for t in (x, dt, z, dy, B, C))
        y, dx, v, gx, gdt, gz, gB, gC = new(D), new(D), new(D), new(D), new(D), new(D), new(S), new(S)
        out, held, dw, db, dA = torch.empty_like(state), torch.empty_like(h), torch.empty_like(taps), torch.empty_like(skip), torch.empty_like(A)
        ctx.hts_short_conv(fx, taps, y, act=hts.ACT_SILU, state_in=state, state_out=out)
        ctx.hts_short_conv_backward(fx, taps, fdy, dx, dw, db=db, act=hts.ACT_SILU, state_in=state)
        states = torch.empty(hts.selective_scan_states(T, N, D, S), device="cuda")
        ctx.hts_selective_scan(fx, fdt, A, fB, fC, v, z=fz, skip=skip, dt_bias=bias, h_in=h, h_out=held, states=states)
        ctx.hts_selective_scan_backward(fx, fdt, A, fB, fC, fdy, states, gx, gdt, gB, gC, dA, z=fz, dz=gz, skip=skip, dt_bias=bias, h_in=h)
        torch.cuda.synchronize()
        results.append([t.clone() for t in (y, dx, v, gx, gdt, gz, gB, gC, out, held, dw, db, dA)])
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), i
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cus", [8, 64])
@pytest.mark.parametrize("T,N,D,S,way", [(700, 1, 200, 16, 2), (300, 5, 130, 13, 0), (129, 2, 34, 8, 1)])
def test_a_range_of_compute_units(hts, dtype, cus, T, N, D, S, way):
    """Fewer units, fewer segments (or none): the workspace is enough, and the values are the definition's."""
    r, way, ty = np.random.default_rng(T + D), dict(WAYS[way]), torch.bfloat16 if dtype == "bf16" else torch.float32
    d, ref = scan_inputs(r, T, N, D, S, 1, way, ty)
    dy = torch.from_numpy(r.normal(size=(T, N, D))).to(ty)
    dy64 = dy.double().numpy()
    rng = hts.CuRangeStream(16, cus)
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32), stream=rng.stream)
    y, held, states = torch.empty(T, N, D, dtype=ty, device="cuda"), torch.empty(N, D, S, device="cuda"), torch.empty(hts.selective_scan_states(T, N, D, S), device="cuda")
    g = {k: torch.empty(T, N, D, dtype=ty, device="cuda") for k in ("dx", "ddt")}
    g["dz"] = torch.empty(T, N, D, dtype=ty, device="cuda") if way["z"] else None
    g.update({k: torch.empty(T, N, 1, S, dtype=ty, device="cuda") for k in ("dB", "dC")}, dA=torch.empty(D, S, device="cuda"), dh_in=torch.empty(N, D, S, device="cuda"))
    dy = dy.cuda()
    torch.cuda.synchronize()                                    # what fills the operands runs on another stream
    forward(hts, ctx, d, way["softplus"], y, h_out=held, states=states)
    ctx.hts_selective_scan_backward(d["x"], d["dt"], d["A"], d["B"], d["C"], dy, states, z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"], softplus=way["softplus"], starts=d["starts"],
                                    lengths=d["lengths"], h_in=d["h_in"], **g)
    torch.cuda.synchronize()
    want, size = (so.scan(**ref, dy=dy64, size=s) for s in (False, True))
    chain = 16 * (T + S) + 12 * 40
    so.near(y.double().cpu().numpy(), want["y"], size["y"], chain, HALF[dtype], "y")
    so.near(held.double().cpu().numpy(), want["h_out"], size["h_out"], chain, HALF["f32"], "h_out")
    for k, v in g.items():
        if v is not None:
            terms = D if k in ("dB", "dC") else T * N if k == "dA" else 0
            so.near(v.double().cpu().numpy(), want[k], size[k], 2 * chain + terms + 32, HALF["f32"] if k in ("dA", "dh_in") else HALF[dtype], k)
    ctx.close()
    rng.close()
