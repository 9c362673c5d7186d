"""Arrays that the gated delta rule's calls write and that share memory with others are refused, on the host: no address is ever read.  areas.hip checks the rule against bytes
written down one by one."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2012_09849_amd import binding as b

HERE = os.path.dirname(os.path.abspath(__file__))
OK, EINVAL, ESHAPE = 0, -1, -2
STEPS = b._Steps
T, N, H, G, K, V = 30, 2, 4, 2, 8, 4
SIZES = {"q": G * K, "k": G * K, "v": H * V, "a": H, "b": H, "y": H * V, "dy": H * V, "dq": G * K, "dk": G * K, "dv": H * V, "da": H, "db": H}
HELD = 4 * N * H * K * V                                  # bytes of the heads' states
DENSE = {"A": 4 * H, "a_bias": 4 * H, "starts": T * N, "lengths": 4 * N, "h_in": HELD, "h_out": HELD, "dh_out": HELD, "dh_in": HELD, "dA": 4 * H, "da_bias": 4 * H, "states": None}
INPUTS = ("q", "k", "v", "a", "b", "A", "a_bias", "starts", "lengths", "h_in")
FORWARD, BACK = ("y", "h_out", "states"), ("dq", "dk", "dv", "da", "db", "dA", "da_bias", "dh_in")


def test_rule(tmp_path):
    exe = str(tmp_path / "areas")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-O2", "-std=c++17", os.path.join(HERE, "areas.hip"), "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", (r.returncode, r.stdout)


@pytest.fixture(scope="module")
def ctx():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_seq_create(0, None, C.byref(h)) == OK
    yield h
    assert lib.hts_seq_destroy(h) == OK


def size(name):
    """Bytes from an array's beginning to its end."""
    if name == "states":
        return 4 * b.delta_rule_states(T, N, H, K, V)
    return DENSE[name] if name in DENSE else 4 * T * N * SIZES[name]


def places(**change):
    at = {n: 0x1000000 * (i + 1) for i, n in enumerate((*SIZES, *DENSE))}
    at.update(change)
    return at


def call(ctx, back, at, wide=None):
    """wide: arrays that are columns of rows of so many entries."""
    steps = lambda n: STEPS(at[n], N * (wide or {}).get(n, SIZES[n]), (wide or {}).get(n, SIZES[n]))  # noqa: E731
    d = b._DeltaDesc(T, N, H, G, K, V, 0, 1, 1, 1.0)
    i = b._DeltaInputs(*[steps(n) if n in SIZES else at[n] for n in INPUTS])
    lib = b.load_library()
    if not back:
        return lib.hts_delta_rule(ctx, C.byref(d), C.byref(i), steps("y"), at["h_out"], at["states"])
    g = b._DeltaGrads(*[steps(n) if n in SIZES else at[n] for n in BACK])
    return lib.hts_delta_rule_backward(ctx, C.byref(d), C.byref(i), steps("dy"), at["dh_out"], at["states"], C.byref(g))


def pairs():
    for back, outs, others in ((False, FORWARD, INPUTS + FORWARD), (True, BACK, INPUTS + ("dy", "dh_out", "states") + BACK)):
        for i, out in enumerate(outs):
            for other in others:
                if other != out and not (other in outs and outs.index(other) < i):
                    yield back, out, other


@pytest.mark.parametrize("back,out,other", list(pairs()))
def test_an_output_that_shares_memory(ctx, back, out, other):
    """At the same address, from its last bytes on, and where the output ends within its first ones; beside each other nothing is refused but the missing workspace."""
    base, step = places()[other], 16 if out == "states" else 4
    for by in (0, (size(other) - 1) // step * step, -((size(out) - 1) // step * step)):
        if {out, other} == {"h_out", "h_in"} and by == 0:
            assert call(ctx, back, places(**{out: base})) == ESHAPE        # the state in its place: only the workspace is missing
            continue
        assert call(ctx, back, places(**{out: base + by})) == EINVAL, by
    for by in ((size(other) + 15) // 16 * 16, -((size(out) + 15) // 16 * 16)):
        assert call(ctx, back, places(**{out: base + by})) == ESHAPE, by


def test_columns_of_wider_arrays(ctx):
    """What a block's products read and write: queries, keys and values beside each other, the gates beside each other, and their gradients; an entry into one another they are refused."""
    C_, base = 2 * G * K + H * V, 0x40000000
    wide = {"q": C_, "k": C_, "v": C_, "dq": C_, "dk": C_, "dv": C_, "a": 2 * H, "b": 2 * H, "da": 2 * H, "db": 2 * H, "y": H * V, "dy": H * V}
    at = places(q=base, k=base + 4 * G * K, v=base + 8 * G * K, a=base + 0x1000000, b=base + 0x1000000 + 4 * H, dq=base + 0x2000000, dk=base + 0x2000000 + 4 * G * K, dv=base + 0x2000000 + 8 * G * K,
                da=base + 0x3000000, db=base + 0x3000000 + 4 * H)
    assert call(ctx, False, at, wide) == ESHAPE and call(ctx, True, at, wide) == ESHAPE
    for name, by in (("dk", -4), ("dv", -4), ("dq", 4), ("db", -4), ("da", 4)):
        assert call(ctx, True, {**at, name: at[name] + by}, wide) == EINVAL, name
    # outputs between the inputs of one wider array
    both = {n: 2 * C_ for n in ("q", "k", "v", "dq", "dk", "dv")}
    at.update(dq=base + 4 * C_, dk=base + 4 * (C_ + G * K), dv=base + 4 * (C_ + 2 * G * K))
    assert call(ctx, True, at, {**wide, **both}) == ESHAPE
    assert call(ctx, True, {**at, "dq": at["dq"] - 4}, {**wide, **both}) == EINVAL
    # the same entries of a wider row, of arrays of other distances
    assert call(ctx, True, {**at, "dv": at["q"] + 4 * C_}, {**wide, **both, "dv": C_}) == EINVAL
