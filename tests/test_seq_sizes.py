"""Shapes that no grid is large enough for, on the host: they are refused by name (HTS_ESHAPE) before anything is launched, so the addresses are never read."""
import ctypes as C

import pytest

from paper_2012_09849_amd import binding as b

OK, ESHAPE = 0, -2
HERE = 0x10000
STEPS = b._Steps


@pytest.fixture(scope="module")
def ctx():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_seq_create(0, None, C.byref(h)) == OK
    yield h
    assert lib.hts_seq_destroy(h) == OK


@pytest.mark.parametrize("T,N,D", [(1 << 30, 1, 1), (1 << 30, 4, 1), (1, 1 << 24, 1 << 10)])
def test_short_conv(ctx, T, N, D):
    d, s = b._ConvDesc(T, N, D, 2, 0, 0), STEPS(HERE, N * D, D)
    assert b.load_library().hts_short_conv(ctx, C.byref(d), s, HERE, None, None, None, None, STEPS(HERE, N * D, D), None) == ESHAPE


@pytest.mark.parametrize("T,N,D,S", [(1, 1 << 24, 64, 1), (2, 1 << 24, 64, 16)])
def test_selective_scan(ctx, T, N, D, S):
    # sequences outermost, so that their distances are within what is taken
    d, s, pair, none = b._ScanDesc(T, N, D, S, 1, 0, 1), STEPS(HERE, D, T * D), STEPS(HERE, S, T * S), STEPS(None, 0, 0)
    inputs = b._ScanInputs(s, s, pair, pair, none, HERE, None, None, None, None, None)
    assert b.load_library().hts_selective_scan(ctx, C.byref(d), C.byref(inputs), s, None, None) == ESHAPE


def test_steps_are_counted_in_32_bits():
    """Chunks go beyond the last step, so that steps near 2^31 would count into the sign: refused."""
    import paper_2012_09849_amd as hts
    most = 1 << 30
    assert hts.short_conv_workspace(most, 1, 1, 2) > 0 and hts.selective_scan_workspace(most, 1, 1, 1) > 0 and hts.selective_scan_states(most, 1, 1, 1) > 0
    for T in (most + 1, (1 << 31) - 1):
        for size in (lambda: hts.short_conv_workspace(T, 1, 1, 2), lambda: hts.selective_scan_workspace(T, 1, 1, 1), lambda: hts.selective_scan_states(T, 1, 1, 1)):
            with pytest.raises(hts.HtsError):
                size()
