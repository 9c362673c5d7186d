"""What the entry points of the sequence memory refuse, on the host: nothing is launched, so no GPU is needed and the addresses are never read."""
import ctypes as C

import pytest
import torch

import paper_2012_09849_amd as hts
from paper_2012_09849_amd import binding as b

OK, EINVAL, ESHAPE = 0, -1, -2
ROWS, STEPS = b._Rows, b._Steps
HERE = 0x10000                        # an address that is a multiple of everything


@pytest.fixture(scope="module")
def ctx():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_seq_create(0, None, C.byref(h)) == OK
    yield h
    assert lib.hts_seq_destroy(h) == OK


def test_context():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_seq_create(-1, None, C.byref(h)) == EINVAL
    assert lib.hts_seq_create(0, None, None) == EINVAL
    assert lib.hts_seq_destroy(None) == EINVAL


@pytest.mark.parametrize("change,code", [(dict(M=0), EINVAL), (dict(N=-1), EINVAL), (dict(K=0), EINVAL), (dict(act=4), EINVAL), (dict(act=-1), EINVAL), (dict(precision=2), ESHAPE),
                                         (dict(K=(1 << 24) + 1), ESHAPE), (dict(desc=None), EINVAL), (dict(x=ROWS(None, 8)), EINVAL), (dict(w=ROWS(HERE + 2, 8)), EINVAL),
                                         (dict(y=ROWS(HERE, 7)), EINVAL), (dict(y=ROWS(HERE, -8)), EINVAL), (dict(x=ROWS(HERE, -1)), EINVAL), (dict(pre=ROWS(HERE, 3)), EINVAL),
                                         (dict(residual=ROWS(HERE + 1, 8)), EINVAL), (dict(bias=HERE + 2), EINVAL), (dict(ctx=None), EINVAL), (dict(x=ROWS(HERE, 1 << 41)), ESHAPE)])
def test_linear(ctx, change, code):
    a = dict(ctx=ctx, M=4, N=8, K=8, precision=0, act=0, x=ROWS(HERE, 8), w=ROWS(HERE, 8), bias=HERE, residual=ROWS(None, 0), y=ROWS(HERE, 8), pre=ROWS(None, 0))
    a.update(change)
    d = b._LinearDesc(a["M"], a["N"], a["K"], a["precision"], a["act"])
    d = None if change.get("desc", 1) is None else C.byref(d)
    assert b.load_library().hts_linear(a["ctx"], d, a["x"], a["w"], a["bias"], a["residual"], a["y"], a["pre"]) == code


@pytest.mark.parametrize("change,code", [(dict(dx=ROWS(None, 0), dw=None, db=None), EINVAL), (dict(dy=ROWS(None, 8)), EINVAL), (dict(act=2, pre=ROWS(None, 0)), EINVAL), (dict(x=ROWS(None, 8)), EINVAL),
                                         (dict(w=ROWS(None, 8)), EINVAL), (dict(dx=ROWS(HERE, 4)), EINVAL), (dict(add=ROWS(HERE + 1, 8)), EINVAL), (dict(dw=HERE + 1), EINVAL),
                                         (dict(act=2, pre=ROWS(HERE, 8)), ESHAPE)])             # the last: no workspace for an activation's gradient
def test_linear_backward(ctx, change, code):
    a = dict(act=0, x=ROWS(HERE, 8), w=ROWS(HERE, 8), pre=ROWS(None, 0), dy=ROWS(HERE, 8), add=ROWS(None, 0), dx=ROWS(HERE, 8), dw=HERE, db=HERE)
    a.update(change)
    d = b._LinearDesc(4, 8, 8, 0, a["act"])
    assert b.load_library().hts_linear_backward(ctx, C.byref(d), *(a[k] for k in ("x", "w", "pre", "dy", "add", "dx", "dw", "db"))) == code


@pytest.mark.parametrize("change,code", [(dict(T=0), EINVAL), (dict(N=0), EINVAL), (dict(D=-4), EINVAL), (dict(act=1), EINVAL), (dict(W=1), ESHAPE), (dict(W=5), ESHAPE), (dict(precision=7), ESHAPE),
                                         (dict(x=STEPS(None, 8, 8)), EINVAL), (dict(w=None), EINVAL), (dict(y=STEPS(HERE, 8, 8)), EINVAL), (dict(y=STEPS(HERE, 12, 8)), EINVAL),
                                         (dict(x=STEPS(HERE, -16, 8)), EINVAL), (dict(lengths=HERE + 1), EINVAL), (dict(T=1 << 30, N=1 << 10), ESHAPE)])
def test_short_conv(ctx, change, code):
    a = dict(T=3, N=2, D=8, W=4, precision=0, act=2, x=STEPS(HERE, 16, 8), w=HERE, bias=None, starts=None, lengths=None, state_in=None, y=STEPS(HERE, 16, 8), state_out=None)
    a.update(change)
    d = b._ConvDesc(*(a[k] for k in ("T", "N", "D", "W", "precision", "act")))
    lib = b.load_library()
    assert lib.hts_short_conv(ctx, C.byref(d), *(a[k] for k in ("x", "w", "bias", "starts", "lengths", "state_in", "y", "state_out"))) == code
    # the same faults of the backward call, with its gradients in y's place
    assert lib.hts_short_conv_backward(ctx, C.byref(d), *(a[k] for k in ("x", "w", "bias", "starts", "lengths", "state_in")), STEPS(HERE, 16, 8), None, a["y"], HERE, None, None) == code


def test_short_conv_backward_more(ctx):
    lib, d, s = b.load_library(), b._ConvDesc(3, 2, 8, 4, 0, 2), STEPS(HERE, 16, 8)
    call = lambda dy=s, dso=None, dx=s, dw=HERE, db=None, dsi=None: lib.hts_short_conv_backward(ctx, C.byref(d), s, HERE, None, None, None, None, dy, dso, dx, dw, db, dsi)  # noqa: E731
    assert call(dw=None) == EINVAL and call(dy=STEPS(None, 0, 0)) == EINVAL and call(dso=HERE, dsi=HERE) == EINVAL and call(db=HERE + 3) == EINVAL
    assert call() == ESHAPE                                     # no workspace


SCAN = dict(T=3, N=2, D=8, S=4, G=2, precision=0, softplus=1)


@pytest.mark.parametrize("change,code", [(dict(T=0), EINVAL), (dict(N=-2), EINVAL), (dict(S=0), EINVAL), (dict(G=0), EINVAL), (dict(softplus=2), EINVAL), (dict(S=65), ESHAPE), (dict(G=3), ESHAPE),
                                         (dict(precision=-1), ESHAPE), (dict(x=STEPS(None, 16, 8)), EINVAL), (dict(dt=STEPS(HERE + 2, 16, 8)), EINVAL), (dict(B=STEPS(None, 16, 8)), EINVAL),
                                         (dict(C=STEPS(HERE, 16, -8)), EINVAL), (dict(A=None), EINVAL), (dict(skip=HERE + 1), EINVAL), (dict(h_in=HERE + 2), EINVAL), (dict(inputs=None), EINVAL)])
def test_selective_scan(ctx, change, code):
    a = dict(SCAN, A=HERE, skip=None, dt_bias=None, starts=None, lengths=None, h_in=None, z=STEPS(None, 0, 0), **{k: STEPS(HERE, 16, 8) for k in ("x", "dt", "B", "C")})
    a.update(change)
    d = b._ScanDesc(*(a[k] for k in SCAN))
    inputs = b._ScanInputs(*(a[k] for k in ("x", "dt", "B", "C", "z", "A", "skip", "dt_bias", "starts", "lengths", "h_in")))
    at = None if change.get("inputs", 1) is None else C.byref(inputs)
    s = STEPS(HERE, 16, 8)
    lib = b.load_library()
    assert lib.hts_selective_scan(ctx, C.byref(d), at, s, None, None) == code
    g = b._ScanGrads(s, s, s, s, STEPS(None, 0, 0), HERE, None, None, None)
    assert lib.hts_selective_scan_backward(ctx, C.byref(d), at, s, None, HERE, C.byref(g)) == code


def test_selective_scan_more(ctx):
    lib, d, s, none = b.load_library(), b._ScanDesc(*SCAN.values()), STEPS(HERE, 16, 8), STEPS(None, 0, 0)
    inputs = b._ScanInputs(s, s, s, s, none, HERE, None, None, None, None, None)
    assert lib.hts_selective_scan(ctx, C.byref(d), C.byref(inputs), STEPS(HERE, 8, 8), None, None) == EINVAL          # overlapping outputs
    assert lib.hts_selective_scan(ctx, C.byref(d), C.byref(inputs), s, None, HERE + 4) == EINVAL                      # states: 16 bytes
    call = lambda states=HERE, dh=None, **k: lib.hts_selective_scan_backward(ctx, C.byref(d), C.byref(inputs), s, dh, states, C.byref(  # noqa: E731
        b._ScanGrads(*({**dict(dx=s, ddt=s, dB=s, dC=s, dz=none, dA=HERE, dskip=None, ddt_bias=None, dh_in=None), **k}.values()))))
    assert call(states=None) == EINVAL and call(dz=s) == EINVAL and call(dA=None) == EINVAL and call(dB=STEPS(HERE, 8, 8)) == EINVAL and call(dh=HERE, dh_in=HERE) == EINVAL
    assert call() == ESHAPE                                     # no workspace


def test_sizes():
    assert hts.linear_workspace(1, 1, 1) >= 0 and hts.short_conv_workspace(1, 1, 1, 2) > 0
    assert hts.selective_scan_states(17, 2, 8, 16) >= 2 * 2 * 8 * 16 and hts.selective_scan_workspace(17, 2, 8, 16) > 0
    for bad in (lambda: hts.linear_workspace(0, 1, 1), lambda: hts.short_conv_workspace(4, 4, 4, 9), lambda: hts.selective_scan_states(4, 4, 4, 99), lambda: hts.selective_scan_workspace(4, 4, 5, 4, G=2)):
        with pytest.raises(hts.HtsError):
            bad()


def test_binding_names_what_is_wrong():
    """Checks of the binding that need no device: every operand has to be a device tensor."""
    with pytest.raises(hts.HtsError, match="x:"):
        b._rows(torch.zeros(2, 2), torch.float32, (2, 2), "x")
    with pytest.raises(hts.HtsError, match="starts:"):
        b._array(torch.zeros(2, 2, dtype=torch.uint8), torch.uint8, (2, 2), "starts")
    with pytest.raises(hts.HtsError, match="y:"):
        b._steps(torch.zeros(2, 2, 2), torch.float32, (2, 2, 2), "y")
    with pytest.raises(hts.HtsError, match="x:"):
        b._precision(torch.zeros(2, dtype=torch.float16), "x")


def test_workspace_is_enough_for_less():
    """A context for T steps of N sequences takes every smaller call: the sizes never fall as T or N grow."""
    for D, S, G in ((1024, 16, 1), (40, 8, 1), (2048, 33, 2)):
        size = lambda T, N: hts.selective_scan_workspace(T, N, D, S, G)  # noqa: E731
        most = size(640, 40)
        for N in range(1, 41):
            for T in (1, 63, 64, 128, 200, 512, 639, 640):
                assert size(T, N) <= size(T + 1, N) and size(T, N) <= size(T, N + 1) and size(T, N) <= most, (D, T, N)
    for f in (lambda T, N: hts.linear_workspace(T * N, 96, 80, act=hts.ACT_SILU), lambda T, N: hts.short_conv_workspace(T, N, 200, 4)):
        assert all(f(T, N) <= f(T + 1, N) and f(T, N) <= f(T, N + 1) for T in range(1, 130, 3) for N in (1, 2, 7, 30))
