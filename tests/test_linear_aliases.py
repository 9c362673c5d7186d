"""Arrays that a matrix product's call writes and that share memory with others are refused, on the host; spans.hip checks the rule against bytes written down one by one."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2012_09849_amd import binding as b

HERE = os.path.dirname(os.path.abspath(__file__))
OK, EINVAL = 0, -1
ROWS = b._Rows
M, N = 6, 8                            # square: K = N
NAMES = ("x", "w", "bias", "residual", "y", "pre")
BACK = ("x", "w", "pre", "dy", "add", "dx", "dw", "db")


def test_rule(tmp_path):
    exe = str(tmp_path / "spans")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-O2", "-std=c++17", os.path.join(HERE, "spans.hip"), "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", (r.returncode, r.stdout)


@pytest.fixture(scope="module")
def ctx():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_seq_create(0, None, C.byref(h)) == OK
    yield h
    assert lib.hts_seq_destroy(h) == OK


def places(names):
    """Addresses far apart; none is ever read, since every call here is refused."""
    return {n: 0x100000 * (i + 1) for i, n in enumerate(names)}


@pytest.mark.parametrize("one,other,by", [("y", "x", 0), ("y", "w", 0), ("y", "bias", 0), ("y", "pre", 0), ("y", "x", 4), ("y", "residual", 4), ("y", "residual", 4 * N), ("pre", "x", 0), ("pre", "w", 8), ("pre", "residual", 0),
                                          ("pre", "bias", -4)])
def test_linear(ctx, one, other, by):
    a = places(NAMES)
    a[one] = a[other] + by
    assert call(ctx, a) == EINVAL


def call(ctx, a):
    d, r = b._LinearDesc(M, N, N, 0, 2), lambda n: ROWS(a[n], N)  # noqa: E731
    return b.load_library().hts_linear(ctx, C.byref(d), r("x"), r("w"), a["bias"], r("residual"), r("y"), r("pre"))


def test_linear_in_the_residuals_place_when_that_is_the_input(ctx):
    a = places(NAMES)
    a["y"] = a["residual"] = a["x"]
    assert call(ctx, a) == EINVAL


def back(ctx, a, act=0):
    d, r = b._LinearDesc(M, N, N, 0, act), lambda n: ROWS(a[n], N)  # noqa: E731
    return b.load_library().hts_linear_backward(ctx, C.byref(d), *(r(n) for n in BACK[:6]), a["dw"], a["db"])


@pytest.mark.parametrize("one,other,by", [("dx", "dy", 0), ("dx", "x", 0), ("dx", "w", 4 * N * (N - 1)), ("dx", "add", 4), ("dx", "dw", 0), ("dx", "db", -4), ("dw", "x", 0), ("dw", "dy", 0), ("dw", "add", 0), ("dw", "w", 0),
                                          ("db", "dy", 4 * (M * N - 1)), ("db", "dw", 4 * (N * N - 1)), ("db", "x", 0), ("db", "add", 0)])
def test_linear_backward(ctx, one, other, by):
    a = places(BACK)
    a[one] = a[other] + by
    assert back(ctx, a) == EINVAL


def test_linear_backward_in_the_place_of_what_is_added_when_that_is_the_gradient(ctx):
    a = places(BACK)
    a["dx"] = a["add"] = a["dy"]
    assert back(ctx, a) == EINVAL
