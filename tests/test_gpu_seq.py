"""The operators of the sequence memory against their definitions in binary64 (seq_oracle.py), through the public entry points.

Tolerances: an output may be off by its own rounding, half a step of its type, and by a count of binary32 roundings of the sum of its terms'
sizes.  Counted are: one for each term of a sum; 16 for a step of a recurrence (step size, its product with A, exp2, three products and sums, the
gate); 12 x 40 for the exponents of a product of decays exp(-x), whose relative error is 12 roundings of x (beyond x = 40 nothing is left of it).
A value that is rounded to bfloat16 on the way to a matrix instruction adds half a step of it to each term.
"""
import numpy as np
import pytest
import torch

import seq_oracle as so

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def hts():
    import paper_2012_09849_amd as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def put(a, dtype=torch.float32):
    """On the GPU in that type, and what arrived there in binary64."""
    if a is None:
        return None, None
    t = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t.cuda(), t.double().numpy()


def inside(shape, dtype, pad, shift, fill=7.0):
    """(whole, view): a view of that shape within a wider array, rows `pad` entries apart, `shift` entries off its start."""
    *lead, k = shape
    whole = torch.full((*lead, k + pad + shift), fill, dtype=dtype, device="cuda")
    return whole, whole[..., shift:shift + k]


def spread(t, pad, shift):
    whole, view = inside(t.shape, t.dtype, pad, shift)
    view.copy_(t)
    return view


def untouched(whole, view_last, shift):
    assert bool((whole[..., :shift] == 7).all()) and bool((whole[..., shift + view_last:] == 7).all())


def host(t):
    return t.double().cpu().numpy()


# ---- matrix product -------------------------------------------------------------------------------------------------
LINEAR_SHAPES = [(1, 1, 1), (1, 512, 512), (16, 2048, 512), (33, 64, 129), (80, 531, 517), (130, 257, 72), (5, 3, 2000), (257, 128, 64), (700, 40, 33), (384, 640, 256),
                 (1030, 136, 200)]


def linear_roundings(K, kind):
    return 2 * K + 8, 0 if kind == "none" else 24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", LINEAR_SHAPES)
@pytest.mark.parametrize("kind,pad,shift", [("none", 0, 0), ("relu", 8, 8), ("silu", 3, 1), ("gelu", 16, 0)])
def test_linear(hts, dtype, M, N, K, kind, pad, shift):
    r, ty = np.random.default_rng(M + N + K), TYPES[dtype]
    (x, x64), (w, w64), (b, b64), (res, res64) = put(r.normal(size=(M, K)), ty), put(r.normal(size=(N, K)) / np.sqrt(K), ty), put(r.normal(size=N)), put(r.normal(size=(M, N)), ty)
    use_b, use_r, use_p = kind != "relu", kind != "silu", kind != "none"
    ctx = hts.SeqContext(hts.linear_workspace(M, N, K, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32, act=getattr(hts, "ACT_" + kind.upper())))
    wide, y = inside((M, N), ty, pad, shift)
    pre = spread(torch.zeros(M, N, dtype=ty, device="cuda"), pad, shift) if use_p else None
    ctx.hts_linear(spread(x, pad, shift), spread(w, pad, shift), y, bias=b if use_b else None, residual=spread(res, pad, shift) if use_r else None, pre=pre,
                   act=getattr(hts, "ACT_" + kind.upper()))
    torch.cuda.synchronize()
    args = (x64, w64, b64 if use_b else None, res64 if use_r else None)
    (want, want_pre), (_, size) = so.linear(*args, kind), so.linear(*args, kind, size=True)
    sums, own = linear_roundings(K, kind)
    if use_p:
        so.near(host(pre), want_pre, size, sums, HALF[dtype], "pre")
    # an activation's slope is at most 1.13; its own roundings, and the exponent's, are of the pre-activation and its square
    so.near(host(y), want, 1.13 * sums * size + own * (np.abs(want_pre) + want_pre ** 2 * (kind != "none")) + (np.abs(res64) if use_r else 0) + np.abs(want), 1, HALF[dtype], "y")
    untouched(wide, N, shift)
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", LINEAR_SHAPES)
@pytest.mark.parametrize("kind,pad,shift", [("none", 0, 0), ("relu", 8, 8), ("silu", 3, 1), ("gelu", 16, 0)])
def test_linear_backward(hts, dtype, M, N, K, kind, pad, shift):
    r, ty = np.random.default_rng(M + 2 * N + K), TYPES[dtype]
    (x, x64), (w, w64), (pre, pre64), (dy, dy64), (add, add64) = (put(r.normal(size=s), ty) for s in ((M, K), (N, K), (M, N), (M, N), (M, K)))
    act = getattr(hts, "ACT_" + kind.upper())
    ctx = hts.SeqContext(hts.linear_workspace(M, N, K, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32, act=act))
    wide, dx = inside((M, K), ty, pad, shift)
    dw, db = torch.full((N, K), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")
    use_add = kind != "relu"
    ctx.hts_linear_backward(spread(x, pad, shift), spread(w, pad, shift), spread(dy, pad, shift), pre=spread(pre, pad, shift) if kind != "none" else None, act=act,
                            add=spread(add, pad, shift) if use_add else None, dx=dx, dw=dw, db=db)
    torch.cuda.synchronize()
    a = add64 if use_add else None
    want, size = (so.linear_grad(x64, w64, pre64, dy64, a, kind, size=s) for s in (False, True))
    # the slope's own roundings grow with the pre-activation's square (an exponent)
    own = 0 if kind == "none" else 16 + 12 * np.abs(pre64).max() ** 2
    rounded = HALF["bf16"] / so.U if dtype == "bf16" and kind != "none" else 0
    so.near(host(dx), want[0], size[0], 2 * N + 8 + own + rounded, HALF[dtype], "dx")
    so.near(host(dw), want[1], size[1], 2 * M + 8 + own + rounded * HALF["bf16"], HALF["f32"], "dw")
    so.near(host(db), want[2], size[2], M + 8 + own, HALF["f32"], "db")
    untouched(wide, K, shift)
    # one output at a time gives the same bits
    for name, out in (("dx", dx), ("dw", dw), ("db", db)):
        alone = torch.empty_like(out).contiguous()
        ctx.hts_linear_backward(x, w, dy, pre=pre if kind != "none" else None, act=act, add=add if use_add else None, **{name: alone})
        torch.cuda.synchronize()
        assert torch.equal(alone, out), name
    ctx.close()


def test_linear_in_place(hts):
    """y may take the residual's place, dx that of what is added; all rows may be one."""
    r = np.random.default_rng(0)
    (x, x64), (w, w64), (res, res64) = put(r.normal(size=(70, 64))), put(r.normal(size=(130, 64))), put(r.normal(size=(70, 130)))
    ctx = hts.SeqContext(hts.linear_workspace(70, 130, 64))
    ctx.hts_linear(x, w, res, residual=res)
    one = torch.empty(70, 130, device="cuda")
    ctx.hts_linear(x[:1].expand(70, 64), w, one)
    torch.cuda.synchronize()
    so.near(host(res), x64 @ w64.T + res64, np.abs(x64) @ np.abs(w64).T + np.abs(res64), 140, HALF["f32"])
    assert torch.equal(one, one[:1].expand(70, 130))
    (dy, dy64), (add, add64) = put(r.normal(size=(70, 130))), put(r.normal(size=(70, 64)))
    ctx.hts_linear_backward(x, w, dy, add=add, dx=add)
    torch.cuda.synchronize()
    so.near(host(add), dy64 @ w64 + add64, np.abs(dy64) @ np.abs(w64) + np.abs(add64), 300, HALF["f32"])
    ctx.close()


def test_linear_nonfinite_stays_in_its_row(hts):
    """An infinity or NaN in a row of x shows in that row of y and nowhere else, also where the reduction ends inside a vector or a tile."""
    for dtype in ("f32", "bf16"):
        for K in (61, 64, 100):
            x, w = torch.randn(90, K, device="cuda").to(TYPES[dtype]), torch.randn(70, K, device="cuda").to(TYPES[dtype])
            clean, y = torch.empty(90, 70, dtype=TYPES[dtype], device="cuda"), torch.empty(90, 70, dtype=TYPES[dtype], device="cuda")
            ctx = hts.SeqContext(hts.linear_workspace(90, 70, K))
            ctx.hts_linear(x, w, clean)
            x[17, K - 1], x[64, 0] = float("nan"), float("inf")
            ctx.hts_linear(x, w, y)
            torch.cuda.synchronize()
            rest = [i for i in range(90) if i not in (17, 64)]
            assert bool(torch.isnan(y[17]).all()) and not bool(torch.isfinite(y[64]).any()) and torch.equal(y[rest], clean[rest])
            ctx.close()


# ---- short convolution ----------------------------------------------------------------------------------------------
CONV_SHAPES = [(1, 1, 1), (1, 48, 1024), (2, 3, 5), (3, 2, 8), (15, 4, 64), (16, 5, 72), (17, 3, 130), (33, 2, 520), (70, 9, 24), (200, 1, 16)]


def sequences(r, T, N, starts, lengths):
    s = (r.random((T, N)) < 0.1).astype(np.uint8) if starts else None
    if starts and T > 4:
        s[0, 0], s[1:4, N - 1], s[T - 1, 0] = 1, 1, 1          # at the first step, one after another, at the last
    n = None
    if lengths:
        n = r.integers(0, T + 1, size=N).astype(np.int32)
        n[0] = T
        if N > 1:
            n[1] = 0
        if N > 2:
            n[2] = 1
        if N > 3:
            n[3] = T + 5                                        # more than there are: all
    return s, n


def spoil(a, lengths):
    """NaN where no step is."""
    if lengths is None:
        return a
    a = a.copy()
    for n, k in enumerate(lengths):
        a[max(0, int(k)):, n] = np.nan
    return a


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D", CONV_SHAPES)
@pytest.mark.parametrize("W,kind,pad,shift,starts,lengths,state", [(4, "silu", 0, 0, True, True, True), (3, "none", 8, 8, True, False, True), (2, "silu", 3, 1, False, True, False),
                                                                   (4, "silu", 16, 0, False, False, False)])
def test_short_conv(hts, dtype, T, N, D, W, kind, pad, shift, starts, lengths, state):
    r, ty = np.random.default_rng(T * N + D + W), TYPES[dtype]
    s, le = sequences(r, T, N, starts, lengths)
    (x, x64), (w, w64), (b, b64), (st, st64) = put(r.normal(size=(T, N, D)), ty), put(r.normal(size=(D, W))), put(r.normal(size=D)), put(r.normal(size=(N, W - 1, D)))
    (dy, dy64), (ds, ds64) = put(r.normal(size=(T, N, D)), ty), put(r.normal(size=(N, W - 1, D)))
    if not state:
        st = st64 = ds = ds64 = None
    (sd, _), (ld, _) = put(s, torch.uint8), put(le, torch.int32)
    act = getattr(hts, "ACT_" + kind.upper())
    ctx = hts.SeqContext(hts.short_conv_workspace(T, N, D, W))
    wide, y = inside((T, N, D), ty, pad, shift)
    out = torch.full((N, W - 1, D), 7.0, device="cuda")
    xs = spread(put(spoil(x64, le), ty)[0], pad, shift)
    ctx.hts_short_conv(xs, w, y, bias=b, act=act, starts=sd, lengths=ld, state_in=st, state_out=out)
    torch.cuda.synchronize()
    want_y, want_out, pre, _ = so.conv(x64, w64, b64, st64, s, le, kind)
    size = W * np.abs(x64).max() * np.abs(w64).max() + np.abs(b64).max() if not state else W * max(np.abs(x64).max(), np.abs(st64).max()) * np.abs(w64).max() + np.abs(b64).max()
    so.near(host(y), want_y, 1.13 * (W + 2) * size + 16 * (np.abs(pre) + pre ** 2), 1, HALF[dtype], "y")
    assert np.array_equal(host(out), want_out), "state_out"
    untouched(wide, D, shift)
    if state:                                                   # the state in its place
        held = st.clone()
        ctx.hts_short_conv(xs, w, y, bias=b, act=act, starts=sd, lengths=ld, state_in=held, state_out=held)
        torch.cuda.synchronize()
        assert torch.equal(held, out)
    wide, dx = inside((T, N, D), ty, pad, shift)
    dw, db, din = torch.full((D, W), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda"), torch.full((N, W - 1, D), 7.0, device="cuda")
    ctx.hts_short_conv_backward(xs, w, spread(put(spoil(dy64, le), ty)[0], pad, shift), dx, dw, db, bias=b, act=act, starts=sd, lengths=ld, state_in=st, dstate_out=ds,
                                dstate_in=din)
    torch.cuda.synchronize()
    want, size = (so.conv_grad(x64, w64, b64, st64, s, le, kind, dy64, ds64, size=z) for z in (False, True))
    # a slope's roundings: its exponent's, of the pre-activation, and what the pre-activation itself is off, times a second derivative of at most 1
    own = 0 if kind == "none" else 24 + 8 * (np.abs(pre).max() ** 2 + (W + 2) * np.abs(pre).max())
    loose = lambda v: v + np.abs(dy64).max() * max(np.abs(w64).max(), np.abs(x64).max()) * (kind != "none")  # noqa: E731
    so.near(host(dx), want[0], loose(size[0]), own + 2 * W + 4, HALF[dtype], "dx")
    so.near(host(dw), want[1], loose(size[1]), own + T * N + 8, HALF["f32"], "dw")
    so.near(host(db), want[2], loose(size[2]), own + T * N + 8, HALF["f32"], "db")
    so.near(host(din), want[3], loose(size[3]), own + 2 * W + 4, HALF["f32"], "dstate_in")
    untouched(wide, D, shift)
    ctx.close()


def test_short_conv_sequences_first_and_others_order(hts):
    """Sequences outermost in memory ([N,T,D] seen as [T,N,D]), and one step at a time with the state handed on: the same values."""
    T, N, D, W = 21, 6, 40, 4
    x, w, b = torch.randn(N, T, D, device="cuda"), torch.randn(D, W, device="cuda"), torch.randn(D, device="cuda")
    starts = (torch.rand(T, N, device="cuda") < 0.2).to(torch.uint8)
    ctx = hts.SeqContext(hts.short_conv_workspace(T, N, D, W))
    whole, held, out = torch.empty(N, T, D, device="cuda"), torch.zeros(N, W - 1, D, device="cuda"), torch.empty(N, W - 1, D, device="cuda")
    ctx.hts_short_conv(x.transpose(0, 1), w, whole.transpose(0, 1), bias=b, act=hts.ACT_SILU, starts=starts, state_out=out)
    for t in range(T):
        y = torch.empty(1, N, D, device="cuda")
        ctx.hts_short_conv(x[:, t][None].contiguous(), w, y, bias=b, act=hts.ACT_SILU, starts=starts[t:t + 1], state_in=held, state_out=held)
        torch.cuda.synchronize()
        assert torch.equal(y[0], whole[:, t])
    assert torch.equal(held, out)
    ctx.close()


# ---- selective scan -------------------------------------------------------------------------------------------------
SCAN_SHAPES = [(1, 1, 1, 1, 1), (1, 32, 64, 16, 1), (2, 3, 6, 3, 2), (5, 2, 16, 8, 1), (15, 2, 17, 16, 1), (16, 1, 48, 13, 1), (17, 3, 34, 16, 2), (33, 4, 130, 5, 1), (40, 2, 24, 20, 3),
               (31, 1, 16, 32, 1), (9, 2, 20, 33, 1), (21, 1, 8, 64, 1), (100, 3, 70, 16, 1), (129, 2, 66, 13, 2)]
WAYS = [dict(z=True, skip=True, bias=True, softplus=True, starts=True, lengths=True, h=True, pad=0, shift=0), dict(z=False, skip=False, bias=False, softplus=False, starts=False, lengths=False, h=False, pad=3, shift=1),
        dict(z=True, skip=True, bias=True, softplus=True, starts=True, lengths=False, h=True, pad=8, shift=8), dict(z=True, skip=False, bias=True, softplus=True, starts=False, lengths=True, h=False, pad=0, shift=0)]


def scan_inputs(r, T, N, D, S, G, way, ty):
    s, le = sequences(r, T, N, way["starts"], way["lengths"])
    arrays = dict(x=r.normal(size=(T, N, D)), dt=r.normal(size=(T, N, D)) * 0.7 if way["softplus"] else r.random((T, N, D)) * 0.5, B=r.normal(size=(T, N, G, S)), C=r.normal(size=(T, N, G, S)),
                  z=r.normal(size=(T, N, D)) if way["z"] else None)
    others = dict(A=-np.exp(r.normal(size=(D, S))), skip=r.normal(size=D) if way["skip"] else None, dt_bias=r.normal(size=D) - 2 if way["bias"] else None,
                  h_in=r.normal(size=(N, D, S)) if way["h"] else None)
    dev, ref = {}, {}
    for k, a in arrays.items():
        t, ref[k] = put(a, ty)
        if t is not None:
            t = put(spoil(ref[k], le), ty)[0]
            flat = t.reshape(T, N, -1)
            dev[k] = spread(flat, way["pad"], way["shift"]).unflatten(2, t.shape[2:])
        else:
            dev[k] = None
    for k, a in others.items():
        dev[k], ref[k] = put(a)
    dev["starts"], dev["lengths"] = put(s, torch.uint8)[0], put(le, torch.int32)[0]
    ref["starts"], ref["lengths"] = s, le
    return dev, dict(ref, softplus=way["softplus"])


def forward(hts, ctx, d, softplus, y, **more):
    ctx.hts_selective_scan(d["x"], d["dt"], d["A"], d["B"], d["C"], y, z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"], softplus=softplus, starts=d["starts"], lengths=d["lengths"], h_in=d["h_in"], **more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D,S,G", SCAN_SHAPES)
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_selective_scan(hts, dtype, T, N, D, S, G, way):
    r, ty, way = np.random.default_rng(T * N + D + S), TYPES[dtype], WAYS[way]
    d, ref = scan_inputs(r, T, N, D, S, G, way, ty)
    (dy, dy64), (dh, dh64) = put(r.normal(size=(T, N, D)), ty), put(r.normal(size=(N, D, S)))
    dy = put(spoil(dy64, ref["lengths"]), ty)[0]
    prec = hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S, G, precision=prec))
    pad, shift = way["pad"], way["shift"]
    wide, y = inside((T, N, D), ty, pad, shift)
    h_out, states = torch.full((N, D, S), 7.0, device="cuda"), torch.empty(hts.selective_scan_states(T, N, D, S, G), device="cuda")
    forward(hts, ctx, d, way["softplus"], y, h_out=h_out, states=states)
    torch.cuda.synchronize()
    want, size = (so.scan(**ref, dy=dy64, dh_out=dh64, size=z) for z in (False, True))
    chain = 16 * (T + S) + 12 * 40
    so.near(host(y), want["y"], size["y"], chain, HALF[dtype], "y")
    so.near(host(h_out), want["h_out"], size["h_out"], chain, HALF["f32"], "h_out")
    untouched(wide, D, shift)
    again, held = torch.empty(T, N, D, dtype=ty, device="cuda"), d["h_in"].clone() if way["h"] else None
    forward(hts, ctx, {**d, "h_in": held}, way["softplus"], again, h_out=held)           # the state in its place, nothing kept for a backward pass
    torch.cuda.synchronize()
    assert torch.equal(again, y) and (held is None or torch.equal(held, h_out))
    g = {k: inside((T, N, D), ty, pad, shift)[1] for k in ("dx", "ddt")}
    g["dz"] = inside((T, N, D), ty, pad, shift)[1] if way["z"] else None
    pairs = {k: inside((T, N, G * S), ty, pad, shift) for k in ("dB", "dC")}
    g.update({k: v[1].unflatten(2, (G, S)) for k, v in pairs.items()})
    g.update(dA=torch.full((D, S), 7.0, device="cuda"), dskip=torch.full((D,), 7.0, device="cuda"), ddt_bias=torch.full((D,), 7.0, device="cuda"), dh_in=torch.full((N, D, S), 7.0, device="cuda"))
    back = lambda out: ctx.hts_selective_scan_backward(d["x"], d["dt"], d["A"], d["B"], d["C"], spread(dy, pad, shift), states, z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"],  # noqa: E731
                                                       softplus=way["softplus"], starts=d["starts"], lengths=d["lengths"], h_in=d["h_in"], dh_out=dh if way["h"] else None, **out)
    back(g)
    torch.cuda.synchronize()
    if not way["h"]:
        want, size = (so.scan(**ref, dy=dy64, size=z) for z in (False, True))
    for k in g:
        if g[k] is not None:
            terms = D if k in ("dB", "dC") else T * N if k in ("dA", "dskip", "ddt_bias") else 0
            so.near(host(g[k]), want[k], size[k], 2 * chain + terms + 32, HALF[dtype] if k in ("dx", "ddt", "dz", "dB", "dC") else HALF["f32"], k)
    for v in pairs.values():
        untouched(v[0], G * S, shift)
    twice = {k: None if v is None else torch.empty_like(v) for k, v in g.items()}
    back(twice)
    torch.cuda.synchronize()
    assert all(v is None or torch.equal(v, twice[k]) for k, v in g.items()), "the same inputs, other bits"
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D,S", [(1, 1024, 16), (16, 200, 16), (3, 130, 7)])
def test_selective_scan_step_by_step(hts, dtype, N, D, S):
    """A prompt in one call, then single steps, against all of it in one call: the same up to the roundings of the state."""
    T, cut, ty = 37, 30, TYPES[dtype]
    d, _ = scan_inputs(np.random.default_rng(D), T, N, D, S, 1, WAYS[2], ty)
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S, 1, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32))
    whole, end, held = torch.empty(T, N, D, dtype=ty, device="cuda"), torch.empty(N, D, S, device="cuda"), d["h_in"].clone()
    forward(hts, ctx, d, True, whole, h_out=end)
    part = lambda a, b: {k: v[a:b] if k in ("x", "dt", "B", "C", "z", "starts") else v for k, v in d.items()}  # noqa: E731
    got = torch.empty(T, N, D, dtype=ty, device="cuda")
    forward(hts, ctx, {**part(0, cut), "h_in": held}, True, got[:cut], h_out=held)
    for t in range(cut, T):
        forward(hts, ctx, {**part(t, t + 1), "h_in": held}, True, got[t:t + 1], h_out=held)
    torch.cuda.synchronize()
    scale = float(end.abs().max())
    assert float((held - end).abs().max()) <= 16 * T * so.U * scale
    assert float((got.float() - whole.float()).abs().max()) <= (2 * HALF[dtype] + 16 * T * so.U) * float(whole.float().abs().max())
    ctx.close()


def test_selective_scan_an_episode_ends_what_is_not_finite(hts):
    """An infinite state and a NaN input of the episode before leave no trace in the next one, forward or backward."""
    T, N, D, S = 40, 2, 20, 16
    d, _ = scan_inputs(np.random.default_rng(4), T, N, D, S, 1, WAYS[0], torch.float32)
    d["lengths"], d["starts"] = None, torch.zeros(T, N, dtype=torch.uint8, device="cuda")
    d["starts"][19] = 1
    for k in ("x", "dt", "B", "C", "z"):
        d[k] = torch.randn_like(d[k])
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S))
    dy = torch.randn(T, N, D, device="cuda")
    dy[:19] = 0

    def both(d):
        y, h, states = torch.empty(T, N, D, device="cuda"), torch.empty(N, D, S, device="cuda"), torch.empty(hts.selective_scan_states(T, N, D, S), device="cuda")
        forward(hts, ctx, d, True, y, h_out=h, states=states)
        g = {k: torch.empty(T, N, D, device="cuda") for k in ("dx", "ddt", "dz")}
        g.update(dB=torch.empty(T, N, 1, S, device="cuda"), dC=torch.empty(T, N, 1, S, device="cuda"), dA=torch.empty(D, S, device="cuda"), dh_in=torch.empty(N, D, S, device="cuda"))
        ctx.hts_selective_scan_backward(d["x"], d["dt"], d["A"], d["B"], d["C"], dy, states, z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"], starts=d["starts"], h_in=d["h_in"], **g)
        torch.cuda.synchronize()
        return y, h, g
    y, h, g = both(d)
    bad = {**d, "h_in": d["h_in"].clone(), "x": d["x"].clone()}
    bad["h_in"][:, ::2], bad["x"][7, :, 1::2] = float("inf"), float("nan")
    y2, h2, g2 = both(bad)
    assert torch.equal(y[19:], y2[19:]) and torch.equal(h, h2) and not bool(torch.isfinite(y2[8:19]).all())
    for k in ("dx", "ddt", "dz"):
        assert torch.equal(g[k][19:], g2[k][19:]), k
    assert bool((g2["dh_in"] == 0).all())
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,D,S,G", [(700, 1, 40, 16, 1), (333, 3, 24, 8, 2), (1000, 1, 70, 33, 1), (260, 2, 18, 20, 1), (512, 2, 64, 16, 1), (257, 16, 16, 16, 1)])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_selective_scan_in_segments(hts, dtype, T, N, D, S, G, way):
    """Few channels and many steps: sequences that are cut into segments, with lengths that end in any of them and episodes that begin in some."""
    r, ty, way = np.random.default_rng(T + N + D), TYPES[dtype], dict(WAYS[way])
    d, ref = scan_inputs(r, T, N, D, S, G, way, ty)
    if way["starts"]:                                           # few, so that states pass through several segments
        s = (r.random((T, N)) < 1.5 / T).astype(np.uint8)
        d["starts"], ref["starts"] = put(s, torch.uint8)[0], s
    for k in ("A",):
        d[k], ref[k] = put(ref[k] * 0.02)
    (dy, dy64), (dh, dh64) = put(r.normal(size=(T, N, D)), ty), put(r.normal(size=(N, D, S)))
    dy = put(spoil(dy64, ref["lengths"]), ty)[0]
    ctx = hts.SeqContext(hts.selective_scan_workspace(T, N, D, S, G, precision=hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32))
    y, held, states = torch.empty(T, N, D, dtype=ty, device="cuda"), torch.zeros(N, D, S, device="cuda"), torch.empty(hts.selective_scan_states(T, N, D, S, G), device="cuda")
    if way["h"]:
        held.copy_(d["h_in"])
    forward(hts, ctx, {**d, "h_in": held}, way["softplus"], y, h_out=held, states=states)               # the state in its place
    torch.cuda.synchronize()
    want, size = (so.scan(**ref, dy=dy64, dh_out=dh64, size=z) for z in (False, True))
    chain = 16 * (T + S) + 12 * 40
    so.near(host(y), want["y"], size["y"], chain, HALF[dtype], "y")
    so.near(host(held), want["h_out"], size["h_out"], chain, HALF["f32"], "h_out")
    g = {k: torch.empty(T, N, D, dtype=ty, device="cuda") for k in ("dx", "ddt")}
    g["dz"] = torch.empty(T, N, D, dtype=ty, device="cuda") if way["z"] else None
    g.update({k: torch.empty(T, N, G, S, dtype=ty, device="cuda") for k in ("dB", "dC")})
    g.update(dA=torch.empty(D, S, device="cuda"), dskip=torch.empty(D, device="cuda"), ddt_bias=torch.empty(D, device="cuda"), dh_in=torch.empty(N, D, S, device="cuda"))
    ctx.hts_selective_scan_backward(d["x"], d["dt"], d["A"], d["B"], d["C"], dy, states, z=d["z"], skip=d["skip"], dt_bias=d["dt_bias"], softplus=way["softplus"], starts=d["starts"],
                                    lengths=d["lengths"], h_in=d["h_in"], dh_out=dh, **g)
    torch.cuda.synchronize()
    for k in g:
        if g[k] is not None:
            terms = D if k in ("dB", "dC") else T * N if k in ("dA", "dskip", "ddt_bias") else 0
            so.near(host(g[k]), want[k], size[k], 2 * chain + terms + 32, HALF[dtype] if k in ("dx", "ddt", "dz", "dB", "dC") else HALF["f32"], k)
    ctx.close()
