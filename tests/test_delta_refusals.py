"""What the entry points of layer norm, the gated delta rule and AdamW refuse, on the host: nothing is launched, so no GPU is needed and the addresses are never read."""
import ctypes as C

import pytest
import torch

import paper_2012_09849_amd as hts
from paper_2012_09849_amd import binding as b

OK, EINVAL, ESHAPE = 0, -1, -2
ROWS, STEPS = b._Rows, b._Steps
HERE = 0x100000                       # an address that is a multiple of everything
NONE = ROWS(None, 0)
INF, NAN = float("inf"), float("nan")


def at(i):
    """Addresses that are far apart."""
    return HERE + i * 0x100000


@pytest.fixture(scope="module")
def ctx():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_seq_create(0, None, C.byref(h)) == OK
    yield h
    assert lib.hts_seq_destroy(h) == OK


@pytest.mark.parametrize("change,code", [(dict(M=0), EINVAL), (dict(F=0), EINVAL), (dict(F=16385), ESHAPE), (dict(M=(1 << 24) + 1), ESHAPE), (dict(precision=2), ESHAPE), (dict(eps=-1e-5), EINVAL),
                                         (dict(eps=NAN), EINVAL), (dict(eps=INF), EINVAL), (dict(x=NONE), EINVAL), (dict(y=NONE), EINVAL), (dict(x=ROWS(at(0) + 2, 8)), EINVAL),
                                         (dict(y=ROWS(at(1), 7)), EINVAL), (dict(y=ROWS(at(0) + 4, 8)), EINVAL), (dict(y=ROWS(at(0), 16)), EINVAL), (dict(w=at(2) + 1), EINVAL),
                                         (dict(b=at(1)), EINVAL), (dict(ctx=None), EINVAL), (dict(desc=None), EINVAL), (dict(x=ROWS(at(0), -8)), EINVAL)])
def test_layer_norm(ctx, change, code):
    a = dict(ctx=ctx, M=4, F=8, precision=0, eps=1e-5, x=ROWS(at(0), 8), w=at(2), b=at(3), y=ROWS(at(1), 8))
    a.update(change)
    d = b._NormDesc(a["M"], a["F"], a["precision"], a["eps"])
    d = None if change.get("desc", 1) is None else C.byref(d)
    assert b.load_library().hts_layer_norm(a["ctx"], d, a["x"], a["w"], a["b"], a["y"]) == code


@pytest.mark.parametrize("change,code", [(dict(dx=NONE, dw=None, db=None), EINVAL), (dict(dy=NONE), EINVAL), (dict(x=NONE), EINVAL), (dict(dx=ROWS(at(1) + 4, 8)), EINVAL), (dict(dx=ROWS(at(1), 9)), EINVAL),
                                         (dict(dx=ROWS(at(2), 8), add=ROWS(at(2) + 16, 8)), EINVAL), (dict(dw=at(0)), EINVAL), (dict(dw=at(4), db=at(4) + 16), EINVAL), (dict(w=at(4)), EINVAL),
                                         (dict(dw=at(4) + 2), EINVAL), (dict(add=ROWS(at(5) + 1, 8)), EINVAL), (dict(), ESHAPE)])          # the last: no workspace
def test_layer_norm_backward(ctx, change, code):
    a = dict(x=ROWS(at(0), 8), w=at(6), dy=ROWS(at(1), 8), add=NONE, dx=ROWS(at(3), 8), dw=at(4), db=at(5))
    a.update(change)
    d = b._NormDesc(4, 8, 0, 1e-5)
    assert b.load_library().hts_layer_norm_backward(ctx, C.byref(d), *(a[k] for k in ("x", "w", "dy", "add", "dx", "dw", "db"))) == code


DELTA = dict(T=30, N=2, H=4, G=2, K=8, V=4, precision=0, normalize=1, softplus=1, scale=1.0)
KEYS, VALUES, GATES = (32, 16), (32, 16), (8, 4)


def delta_inputs(**change):
    a = dict(q=STEPS(at(0), *KEYS), k=STEPS(at(1), *KEYS), v=STEPS(at(2), *VALUES), a=STEPS(at(3), *GATES), b=STEPS(at(4), *GATES), A=at(5), a_bias=None, starts=None, lengths=None, h_in=None)
    a.update(change)
    return b._DeltaInputs(*a.values())


def delta_grads(**change):
    a = dict(dq=STEPS(at(10), *KEYS), dk=STEPS(at(11), *KEYS), dv=STEPS(at(12), *VALUES), da=STEPS(at(13), *GATES), db=STEPS(at(14), *GATES), dA=at(15), da_bias=None, dh_in=None)
    a.update(change)
    return b._DeltaGrads(*a.values())


@pytest.mark.parametrize("change,code", [(dict(T=0), EINVAL), (dict(N=-1), EINVAL), (dict(H=0), EINVAL), (dict(G=0), EINVAL), (dict(G=3), ESHAPE), (dict(K=129), ESHAPE), (dict(K=0), EINVAL), (dict(V=0), EINVAL),
                                         (dict(V=(1 << 16) + 1), ESHAPE), (dict(precision=5), ESHAPE), (dict(normalize=2), EINVAL), (dict(softplus=-1), EINVAL), (dict(scale=NAN), EINVAL),
                                         (dict(scale=INF), EINVAL), (dict(T=(1 << 30) + 1), ESHAPE), (dict(T=1 << 30, N=1 << 20, H=1 << 10, G=1), ESHAPE), (dict(q=STEPS(None, 8, 8)), EINVAL),
                                         (dict(k=STEPS(at(1) + 2, *KEYS)), EINVAL), (dict(v=STEPS(at(2), -16, 8)), EINVAL), (dict(a=STEPS(None, 0, 0)), EINVAL), (dict(b=STEPS(at(4), 1 << 25, 4)), ESHAPE),
                                         (dict(A=None), EINVAL), (dict(a_bias=at(6) + 1), EINVAL), (dict(h_in=at(6) + 2), EINVAL), (dict(lengths=at(6) + 1), EINVAL), (dict(inputs=None), EINVAL), (dict(ctx=None), EINVAL)])
def test_delta_rule(ctx, change, code):
    sizes = {**DELTA, **{k: v for k, v in change.items() if k in DELTA}}
    given = delta_inputs(**{k: v for k, v in change.items() if k not in DELTA and k not in ("inputs", "ctx")})
    d, i = b._DeltaDesc(*sizes.values()), None if "inputs" in change else C.byref(given)
    h = None if "ctx" in change else ctx
    lib, y = b.load_library(), STEPS(at(7), *VALUES)
    assert lib.hts_delta_rule(h, C.byref(d), i, y, None, None) == code
    assert lib.hts_delta_rule_backward(h, C.byref(d), i, STEPS(at(8), *VALUES), None, at(9), C.byref(delta_grads())) == code


def test_delta_rule_more(ctx):
    lib, d, i = b.load_library(), b._DeltaDesc(*DELTA.values()), delta_inputs()
    call = lambda y=STEPS(at(7), *VALUES), h=None, states=None: lib.hts_delta_rule(ctx, C.byref(d), C.byref(i), y, h, states)  # noqa: E731
    assert call() == ESHAPE                                                           # no workspace
    assert call(y=STEPS(None, 0, 0)) == EINVAL and call(y=STEPS(at(7), 16, 16)) == EINVAL and call(y=STEPS(at(2), *VALUES)) == EINVAL
    assert call(states=at(9) + 4) == EINVAL and call(states=at(9), h=at(9)) == EINVAL and call(h=at(9) + 1) == EINVAL
    back = lambda dy=STEPS(at(8), *VALUES), dh=None, states=at(9), **k: lib.hts_delta_rule_backward(ctx, C.byref(d), C.byref(i), dy, dh, states, C.byref(delta_grads(**k)))  # noqa: E731
    assert back() == ESHAPE
    assert back(states=None) == EINVAL and back(dy=STEPS(None, 0, 0)) == EINVAL and back(dA=None) == EINVAL and back(dq=STEPS(at(0), *KEYS)) == EINVAL
    assert back(dk=STEPS(at(10), *KEYS)) == EINVAL and back(dv=STEPS(at(8), *VALUES)) == EINVAL and back(da=STEPS(at(13), 4, 4)) == EINVAL
    assert back(dh=at(20), dh_in=at(20)) == EINVAL and back(da_bias=at(15)) == EINVAL and back(dh_in=at(9)) == EINVAL and back(dh_in=at(20) + 2) == EINVAL


def test_sizes():
    assert hts.layer_norm_workspace(1, 1) > 0 and hts.delta_rule_states(65, 2, 3, 8, 4) >= 2 * 2 * 3 * (8 * 4 + 64 * 4)
    for bad in (lambda: hts.layer_norm_workspace(0, 4), lambda: hts.layer_norm_workspace(4, 20000), lambda: hts.delta_rule_workspace(4, 4, 4, 3, 8, 8), lambda: hts.delta_rule_states(4, 4, 4, 200, 8)):
        with pytest.raises(hts.HtsError):
            bad()
    # a context for T steps of N sequences, or M rows, takes every smaller call
    for size in (lambda T, N: hts.delta_rule_workspace(T, N, 3, 1, 33, 40), lambda T, N: hts.delta_rule_states(T, N, 3, 33, 40), lambda T, N: hts.layer_norm_workspace(T * N, 300)):
        assert all(size(T, N) <= size(T + 1, N) and size(T, N) <= size(T, N + 1) for T in range(1, 300, 7) for N in (1, 2, 7, 30))


def tensor(**change):
    a = dict(p=at(0), g=at(1), m=at(2), v=at(3), m_scale=None, v_scale=None, copy=None, n=100, weight_decay=0.0, lr_scale=1.0, grad_precision=0, bits=32)
    a.update(change)
    return b._AdamWTensorC(*a.values())


EIGHT = dict(bits=8, m_scale=at(4), v_scale=at(5))


@pytest.mark.parametrize("tensors,code", [([], EINVAL), ([dict(p=None)], EINVAL), ([dict(g=None)], EINVAL), ([dict(m=None)], EINVAL), ([dict(v=None)], EINVAL), ([dict(n=0)], EINVAL), ([dict(n=(1 << 34) + 1)], EINVAL),
                                          ([dict(bits=16)], EINVAL), ([dict(grad_precision=2)], ESHAPE), ([dict(p=at(0) + 2)], EINVAL), ([dict(m=at(2) + 1)], EINVAL), ([dict(copy=at(6) + 1)], EINVAL),
                                          ([dict(bits=8)], EINVAL), ([dict(EIGHT, v_scale=None)], EINVAL), ([dict(EIGHT, m_scale=at(4) + 2)], EINVAL), ([dict(weight_decay=NAN)], EINVAL),
                                          ([dict(weight_decay=-1.0)], EINVAL), ([dict(lr_scale=INF)], EINVAL), ([dict(m=at(0) + 200)], EINVAL), ([dict(g=at(0))], EINVAL), ([dict(copy=at(1) + 8)], EINVAL),
                                          ([dict(), dict()], EINVAL), ([dict(), dict(p=at(8), g=at(2) + 396, m=at(9), v=at(10))], EINVAL), ([dict(EIGHT, v_scale=at(4) + 0)], EINVAL)])
def test_adamw_plans(tensors, code):
    lib, h = b.load_library(), C.c_void_p()
    # (lengths are looked at after addresses: an array that long meets the next one)
    table = (b._AdamWTensorC * max(1, len(tensors)))(*[tensor(**t) for t in tensors])
    rc = lib.hts_adamw_create(table, len(tensors), None, C.byref(h))
    assert rc == (ESHAPE if tensors and tensors[0].get("n", 0) > 1 << 34 else code) and not h.value


def test_adamw_more():
    lib, h = b.load_library(), C.c_void_p()
    assert lib.hts_adamw_create(None, 1, None, C.byref(h)) == EINVAL and lib.hts_adamw_create(C.byref(tensor()), 1, None, None) == EINVAL and lib.hts_adamw_create(C.byref(tensor()), -1, None, C.byref(h)) == EINVAL
    assert lib.hts_adamw_destroy(None) == EINVAL and lib.hts_adamw_step(None, C.byref(hts.AdamWHParams()), C.byref(C.c_int64(0)), None) == EINVAL
    assert hts.adamw_scales(1) == 1 and hts.adamw_scales(256) == 1 and hts.adamw_scales(257) == 2
    with pytest.raises(hts.HtsError):
        hts.AdamW([hts.AdamWTensor(torch.zeros(3), torch.zeros(3), torch.zeros(3), torch.zeros(3))])
