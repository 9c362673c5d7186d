"""The gated delta rule and its gradients against the definition in binary64 (delta_oracle.py, whose `allowed` says how far they may be from it), through the
public entry points."""
import numpy as np
import pytest
import torch

import delta_oracle as do
import seq_oracle as so
from test_gpu_seq import HALF, TYPES, hts, host, inside, put, spread, untouched  # noqa: F401

pytestmark = pytest.mark.gpu


class Case:
    """Inputs, their values in binary64, and a context."""

    def __init__(self, hts, dtype, T, N, G, H, K, V, seed=0, pad=0, shift=0, starts=0.0, lengths=None, softplus=True, normalize=True, bias=True, state=True, workspace=None):  # noqa: F811
        r, self.ty, self.dtype, self.hts = np.random.default_rng(seed + T + 3 * N + 5 * K + 7 * V), TYPES[dtype], dtype, hts
        self.shape = T, N, G, H, K, V
        n = lambda *s: r.normal(size=s)  # noqa: E731
        silu = lambda x: x / (1 + np.exp(-x))  # noqa: E731
        size = (1.0 if normalize else K ** -0.5)
        given = {"q": silu(n(T, N, G, K)) * size, "k": silu(n(T, N, G, K)) * size, "v": n(T, N, H, V), "a": n(T, N, H) if softplus else np.abs(n(T, N, H)) * 0.1, "b": n(T, N, H), "dy": n(T, N, H, V)}
        self.at, self.wide = {}, {}
        for name, x in given.items():
            t, self.wide[name] = put(x, self.ty)
            flat = spread(t.flatten(2), pad, shift)
            self.at[name] = flat.unflatten(2, t.shape[2:]) if t.dim() == 4 else flat
        for name, x in (("A", -(0.5 + 6 * r.random(H)) if softplus else -np.ones(H)), ("a_bias", -2 + n(H) if bias and softplus else None), ("h_in", n(N, H, K, V) if state else None),
                        ("dh_out", n(N, H, K, V) if state else None)):
            self.at[name], self.wide[name] = put(x)
        s = (r.random((T, N)) < starts).astype(np.uint8) if starts else None
        self.at["starts"], self.wide["starts"] = (torch.from_numpy(s).cuda(), s) if starts else (None, None)
        self.set_lengths(lengths)
        self.more = {"scale": float(np.float32(K ** -0.5)), "normalize": normalize, "softplus": softplus}
        self.precision = hts.PRECISION_BF16 if dtype == "bf16" else hts.PRECISION_FP32
        self.ctx = hts.SeqContext(hts.delta_rule_workspace(T, N, H, G, K, V, precision=self.precision) if workspace is None else workspace)
        self.pad, self.shift = pad, shift

    def set_lengths(self, lengths):
        self.wide["lengths"] = None if lengths is None else np.asarray(lengths, dtype=np.int32)
        self.at["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")

    def new(self, *shape):
        """An output between sevens."""
        whole, view = inside((*shape[:2], int(np.prod(shape[2:]))), self.ty, self.pad, self.shift)
        self.whole.append((whole, view.shape[2]))
        return view.unflatten(2, shape[2:])

    def run(self, gradients=True, ctx=None):
        T, N, G, H, K, V = self.shape
        ctx, at, self.whole = ctx or self.ctx, self.at, []
        ins = [at[c] for c in ("q", "k", "v", "a", "b", "A")]
        seq = dict(a_bias=at["a_bias"], starts=at["starts"], lengths=at["lengths"], h_in=at["h_in"], **self.more)
        out = {"y": self.new(T, N, H, V), "h_out": torch.full((N, H, K, V), 7.0, device="cuda")}
        states = torch.full((self.hts.delta_rule_states(T, N, H, K, V),), float("nan"), device="cuda") if gradients else None
        ctx.hts_delta_rule(*ins, out["y"], h_out=out["h_out"], states=states, **seq)
        if gradients:
            g = {"dq": self.new(T, N, G, K), "dk": self.new(T, N, G, K), "dv": self.new(T, N, H, V), "da": self.new(T, N, H), "db": self.new(T, N, H)}
            g["da"], g["db"] = (g[c].flatten(2) for c in ("da", "db"))
            g.update(dA=torch.full((H,), 7.0, device="cuda"), da_bias=torch.full((H,), 7.0, device="cuda"), dh_in=torch.full((N, H, K, V), 7.0, device="cuda"))
            ctx.hts_delta_rule_backward(*ins, at["dy"], states, dh_out=at["dh_out"], **g, **seq)
            out.update(g)
        torch.cuda.synchronize()
        for whole, k in self.whole:
            untouched(whole, k, self.shift)
        return out

    def oracle(self, gradients=True):
        wide = {c: self.wide[c] for c in ("q", "k", "v", "a", "b", "A", "a_bias", "starts", "lengths", "h_in")}
        want, sizes = do.delta(**wide, **self.more, **({"dy": self.wide["dy"], "dh_out": self.wide["dh_out"]} if gradients else {}))
        T, N, G, H, K, V = self.shape
        x = self.wide["a"] + (0 if self.wide["a_bias"] is None else self.wide["a_bias"])
        step = np.logaddexp(0, x) if self.more["softplus"] else x
        off = do.allowed(sizes, {"y": (T, N, H, V), "dv": (T, N, H, V), "dq": (T, N, G, K), "db": (T, N, H)}, T, K, self.wide["A"], np.exp(step * self.wide["A"]), self.wide["dy"], self.more["scale"], self.more["normalize"], self.wide["k"], self.wide["q"])
        if gradients:
            off["dA"] = (off.pop("dlog") * np.abs(step)).sum((0, 1))
        return want, off

    def check(self, gradients=True):
        got = self.run(gradients)
        want, off = self.oracle(gradients)
        for name in got:
            half = HALF["f32" if got[name].dtype is torch.float32 else self.dtype]
            so.near(host(got[name]), want[name], off[name] / so.U, 1, half, name)
        return got


# steps around a chunk's; one of everything; widths that are multiples of nothing and the largest
SHAPES = [(1, 1, 1, 1, 1, 1), (1, 3, 2, 4, 128, 70), (2, 2, 1, 1, 5, 3), (5, 4, 2, 2, 64, 64), (16, 2, 1, 3, 33, 130), (17, 2, 1, 1, 16, 16), (63, 1, 1, 2, 37, 53), (64, 2, 1, 1, 32, 32),
          (65, 2, 2, 2, 64, 33), (130, 1, 1, 1, 128, 128), (200, 2, 1, 4, 100, 20), (129, 3, 3, 6, 24, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,G,H,K,V", SHAPES)
@pytest.mark.parametrize("pad,shift,starts", [(0, 0, 0.0), (3, 1, 0.1)])
def test_values_and_gradients(hts, dtype, T, N, G, H, K, V, pad, shift, starts):  # noqa: F811
    c = Case(hts, dtype, T, N, G, H, K, V, pad=pad, shift=shift, starts=starts)
    c.check()
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,G,H,K,V", [(70, 1, 1, 1, 16, 1100), (20, 1000, 1, 1, 8, 8), (3, 3000, 1, 2, 4, 4), (66, 2, 1, 40, 12, 8)])
def test_many(hts, dtype, T, N, G, H, K, V):  # noqa: F811
    """Many tiles of values, many sequences, many heads of one group."""
    c = Case(hts, dtype, T, N, G, H, K, V, starts=0.05)
    c.check()
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,G,H,K,V,starts", [(800, 1, 1, 1, 16, 24, 0.0), (1100, 2, 1, 2, 40, 40, 0.002), (1600, 1, 1, 1, 128, 128, 0.0), (900, 1, 1, 1, 64, 33, 0.01)])
def test_long(hts, dtype, T, N, G, H, K, V, starts):  # noqa: F811
    """Long sequences of few heads are worked on in segments at the same time: sequences that end in the first one, in a later one and at one's end among them; states of chunks."""
    for lengths in (None, [T // 2 + 3] * N, [130] * N, [0] * N, [768] * N):
        c = Case(hts, dtype, T, N, G, H, K, V, starts=starts, lengths=lengths)
        got, plain = c.run(), c.run(False)
        want, off = c.oracle()
        for name in got:
            so.near(host(got[name]), want[name], off[name] / so.U, 1, HALF["f32" if got[name].dtype is torch.float32 else dtype], name)
        assert torch.equal(got["y"], plain["y"]) and torch.equal(got["h_out"], plain["h_out"])
        # ... and the state at the end in the place of the one at the beginning, which every segment's is made of
        state, y = c.at["h_in"].clone(), torch.empty(T, N, H, V, dtype=c.ty, device="cuda")
        at = c.at
        c.ctx.hts_delta_rule(*(at[n] for n in ("q", "k", "v", "a", "b", "A")), y, a_bias=at["a_bias"], starts=at["starts"], lengths=at["lengths"], h_in=state, h_out=state, **c.more)
        torch.cuda.synchronize()
        assert torch.equal(got["y"], y) and torch.equal(got["h_out"], state)
        c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [4, 140])
def test_lengths(hts, dtype, T):  # noqa: F811
    """Sequences of no steps, of one, up to and past a chunk's end, fewer than none and more than all; what lies behind is not read, outputs there are zeros, states stay."""
    lengths = [0, 1, min(T, 63), min(T, 64), min(T, 65), T, -3, T + 9]
    c = Case(hts, dtype, T, len(lengths), 1, 2, 20, 40, starts=0.05, lengths=lengths)
    for n, length in enumerate(lengths):
        for name in ("q", "k", "v", "a", "b", "dy"):
            c.at[name][max(0, length):, n] = float("nan")
    got = c.check()
    for n, length in enumerate(lengths):
        length = max(0, length)
        for name in ("y", "dq", "dk", "dv", "da", "db"):
            assert bool((got[name][length:, n] == 0).all()), name
        if length == 0:
            assert torch.equal(got["h_out"][n], c.at["h_in"][n]) and torch.equal(got["dh_in"][n], c.at["dh_out"][n])
    c.ctx.close()


@pytest.mark.parametrize("begins", [[0], [63], [64], [5, 6, 7], [0, 64, 128], list(range(70))])
def test_starts(hts, begins):  # noqa: F811
    c = Case(hts, "f32", 131, 2, 1, 2, 16, 33, starts=0.5)
    s = np.zeros((131, 2), dtype=np.uint8)
    s[begins, 0] = 1
    c.wide["starts"], c.at["starts"] = s, torch.from_numpy(s).cuda()
    got = c.check()
    assert bool((got["da"][begins, 0] == 0).all())
    if 0 in begins:
        assert bool((got["dh_in"][0] == 0).all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("softplus,normalize,bias,state", [(False, True, False, False), (True, False, True, True), (True, True, False, False)])
def test_options(hts, dtype, softplus, normalize, bias, state):  # noqa: F811
    for T in (3, 100):
        c = Case(hts, dtype, T, 2, 2, 2, 48, 17, softplus=softplus, normalize=normalize, bias=bias, state=state)
        c.check()
        c.ctx.close()


def test_decays(hts):  # noqa: F811
    """Decays from none at all to ones that leave nothing of binary32, beside each other in a chunk: products over many steps keep the small ones' digits."""
    c = Case(hts, "f32", 128, 2, 1, 2, 16, 16, softplus=False)
    a = np.abs(np.random.default_rng(3).normal(size=(128, 2, 2))) * 0.01
    a[::9] = 60.0
    a[4::31] = 200.0
    a[5::40] = np.inf
    a[2::7] = 0.0
    c.at["a"], c.wide["a"] = put(a)
    c.wide["a"] = np.minimum(c.wide["a"], 800.0)               # (the oracle's exp is 0 there too, and 0 times it no NaN)
    got = c.run()
    want, off = c.oracle()
    for name in got:
        if name == "dA":
            continue                                           # (the last factor of an infinite step)
        so.near(host(got[name]), want[name], off[name] / so.U, 1, HALF["f32"], name)
    c.ctx.close()


def test_strengths_of_nothing_and_of_one(hts):  # noqa: F811
    c = Case(hts, "f32", 90, 1, 1, 2, 16, 16)
    b = np.random.default_rng(4).normal(size=(90, 1, 2))
    b[::3], b[1::5] = -200.0, 200.0
    c.at["b"], c.wide["b"] = put(b)
    c.check()
    c.ctx.close()


def test_keys_alike(hts):  # noqa: F811
    """The same key at every step, and keys of nothing but zeros: the substitution's largest factors."""
    c = Case(hts, "f32", 128, 2, 1, 1, 8, 8)
    k = np.tile(c.wide["k"][:1], (128, 1, 1, 1))
    k[:, 1] = 0
    c.at["k"], c.wide["k"] = put(k)
    b = np.full((128, 2, 1), 9.0)
    c.at["b"], c.wide["b"] = put(b)
    c.check()
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_states_and_pieces(hts, dtype):  # noqa: F811
    """h_out in h_in's place; a sequence in pieces, down to single steps, is the whole one."""
    T, N, G, H, K, V = 100, 2, 1, 2, 32, 40
    c = Case(hts, dtype, T, N, G, H, K, V, starts=0.02)
    want, off = c.oracle(False)
    state, y = c.at["h_in"].clone(), torch.empty(T, N, H, V, dtype=c.ty, device="cuda")
    for first, last in ((0, 1), (1, 2), (2, 70), (70, 75), (75, 76), (76, 100)):
        part = {n: c.at[n][first:last] for n in ("q", "k", "v", "a", "b")}
        starts = c.at["starts"][first:last].contiguous()
        c.ctx.hts_delta_rule(*part.values(), c.at["A"], y[first:last], a_bias=c.at["a_bias"], starts=starts, h_in=state, h_out=state, **c.more)
    torch.cuda.synchronize()
    so.near(host(y), want["y"], off["y"] / so.U, 2, HALF[dtype], "y")
    so.near(host(state), want["h_out"], off["h_out"] / so.U, 2, HALF["f32"], "h_out")
    c.ctx.close()


@pytest.mark.parametrize("T", [12, 130])
def test_not_finite(hts, T):  # noqa: F811
    """What is not finite reaches what sees it and nothing else: not the steps before it, not the episodes after it, not other sequences, nor, of the values, other heads."""
    N, G, H, K, V = 3, 1, 2, 16, 40
    clean = Case(hts, "f32", T, N, G, H, K, V, starts=0.5)
    s = np.zeros((T, N), dtype=np.uint8)
    s[T // 2] = 1
    s[:, 2] = 0
    s[0, 2] = 1
    clean.at["starts"] = torch.from_numpy(s).cuda()
    base = clean.run(T > 64)
    at = T // 4
    for name, value in (("v", np.nan), ("v", np.inf), ("k", np.nan), ("k", -np.inf), ("q", np.nan), ("b", np.nan), ("a", np.nan), ("dy", np.nan), ("dy", np.inf)):
        if name == "dy" and T <= 64:
            continue
        kept = clean.at[name].clone()
        x = clean.at[name][at, 0].flatten()
        x[3 if name in ("v", "dy") else 0] = float(value)       # (a and b: of head 0)
        clean.at[name][at, 0] = x.view(clean.at[name][at, 0].shape)
        got = clean.run(T > 64)
        mine = "h_out" if T // 2 == 0 else None
        assert mine is None
        assert torch.equal(got["y"][:at, 0], base["y"][:at, 0]) or name == "dy" or np.allclose(host(got["y"][:at, 0]), host(base["y"][:at, 0]), atol=1e-5), name
        assert bool(got["y"][T // 2:].isfinite().all()) and bool(got["y"][:, 1:].isfinite().all()) and bool(got["h_out"].isfinite().all()), name
        if name != "dy":
            assert not bool(got["y"][at, 0].isfinite().all()), name
        if name == "v":
            assert bool(got["y"][:, 0, 1].isfinite().all())
        if T > 64:
            for g in ("dq", "dk", "dv", "da", "db"):
                assert bool(got[g][T // 2:].isfinite().all()) and bool(got[g][:, 1:].isfinite().all()), (name, g)
                assert np.allclose(host(got[g][T // 2:, 0]), host(base[g][T // 2:, 0]), atol=1e-4), (name, g)
            assert bool(got["dh_in"][1:].isfinite().all())
            if name == "dy":
                assert not bool(got["dv"][at, 0].isfinite().all()) and not bool(got["dh_in"][0].isfinite().all())
                for g in ("dq", "dk", "dv"):
                    assert bool(got[g][at + 1:, 0].isfinite().all()), g
        clean.at[name].copy_(kept)
    # a state that is not finite, of a sequence whose first step begins an episode, and of one without steps
    clean.at["h_in"][2] = float("nan")
    got = clean.run(T > 64)
    assert bool(got["y"].isfinite().all()) and bool(got["h_out"].isfinite().all())
    if T > 64:
        assert all(bool(got[g].isfinite().all()) for g in ("dq", "dk", "dv", "da", "db", "dA", "da_bias", "dh_in")) and bool((got["dh_in"][2] == 0).all())
    clean.set_lengths([T, T, 0])
    got = clean.run(T > 64)
    assert bool(got["h_out"][2].isnan().all()) and bool(got["y"].isfinite().all())
    if T > 64:
        assert all(bool(got[g].isfinite().all()) for g in ("dq", "dk", "dv", "da", "db", "dA", "da_bias", "dh_in"))
    clean.ctx.close()


@pytest.mark.parametrize("T", [1, 16, 20])
@pytest.mark.parametrize("normalize", [True, False])
def test_squares_that_are_not_finite(hts, T, normalize):  # noqa: F811
    """A key or query of finite entries whose square is beyond binary32 is none: the same of a few steps as of many."""
    c = Case(hts, "bf16", T, 2, 1, 2, 16, 40, normalize=normalize)
    for name in ("k", "q"):
        kept = c.at[name].clone()
        c.at[name][T // 2, 0] = 1e20
        got = c.run()
        c.at[name].copy_(kept)
        assert bool(got["y"][:T // 2].isfinite().all()) and bool(got["y"][:, 1].isfinite().all()) and bool(got["h_out"][1].isfinite().all()), name
        assert bool(got["y"][T // 2, 0].isnan().all()), name
        if name == "k":
            assert bool(got["y"][T // 2:, 0].isnan().all()) and bool(got["h_out"][0].isnan().all())
        else:
            assert bool(got["y"][T // 2 + 1:].isfinite().all()) and bool(got["h_out"].isfinite().all())
    c.ctx.close()


def test_not_finite_in_segments(hts):  # noqa: F811
    """A long sequence in segments: what one makes of the state before it is not multiplied by what is not finite where an episode begins in it."""
    c = Case(hts, "f32", 900, 1, 1, 1, 16, 40, starts=0.5)
    s = np.zeros((900, 1), dtype=np.uint8)
    s[[0, 500, 700]] = 1
    c.at["starts"] = torch.from_numpy(s).cuda()
    c.at["h_in"][:] = float("inf")
    base = c.run(False)
    assert bool(base["y"].isfinite().all()) and bool(base["h_out"].isfinite().all())
    for name in ("v", "k", "a"):
        kept = c.at[name].clone()
        c.at[name][130] = float("nan")
        got = c.run(False)
        c.at[name].copy_(kept)
        assert bool(got["y"][:130].isfinite().all()) and bool(got["y"][130:500].isnan().all()) and bool(got["y"][500:].isfinite().all()), name
        assert np.allclose(host(got["y"][500:]), host(base["y"][500:]), atol=1e-5) and bool(got["h_out"].isfinite().all())
    s[0] = 0
    c.at["starts"] = torch.from_numpy(s).cuda()
    got = c.run(False)
    assert not bool(got["y"][:500].isfinite().any()) and bool(got["y"][500:].isfinite().all())
    c.ctx.close()


def test_streams_of_some_units(hts):  # noqa: F811
    """The same bits on a range of compute units, in segments and not."""
    for T, N in ((900, 1), (100, 3)):
        c = Case(hts, "bf16", T, N, 1, 2, 32, 32)
        want = c.run()
        part = hts.CuRangeStream(0, 64)
        ctx = hts.SeqContext(hts.delta_rule_workspace(T, N, 2, 1, 32, 32, precision=hts.PRECISION_BF16), stream=part.stream)
        torch.cuda.synchronize()
        got = c.run(ctx=ctx)
        assert all(torch.equal(want[n], got[n]) for n in want)
        ctx.close()
        part.close()
        c.ctx.close()


def test_one_row_for_all_and_far_apart(hts):  # noqa: F811
    """Strides of nothing (the same queries, keys and gates at every step of every sequence), and sequences that lie between another array's."""
    T, N, G, H, K, V = 70, 3, 1, 2, 24, 20
    c = Case(hts, "f32", T, N, G, H, K, V)
    for name in ("q", "k", "a", "b"):
        one = c.at[name][:1, :1].clone()
        c.at[name] = one.expand(T, N, *one.shape[2:])
        c.wide[name] = c.at[name].double().cpu().numpy()
    by_sequence = torch.randn(N, T, 2, H, V, device="cuda")
    c.at["v"] = by_sequence[:, :, 1].transpose(0, 1)
    c.wide["v"] = c.at["v"].double().cpu().numpy()
    c.check()
    c.ctx.close()


def test_bits(hts):  # noqa: F811
    """The same bits again, in a context with more workspace than needed, and whatever the workspace held."""
    c = Case(hts, "bf16", 150, 2, 1, 2, 64, 64, starts=0.05)
    first = c.run()
    other = hts.SeqContext(hts.delta_rule_workspace(400, 4, 3, 1, 128, 128, precision=hts.PRECISION_BF16))
    for _ in range(2):
        again = c.run(ctx=other)
        assert all(torch.equal(first[n], again[n]) for n in first)
    other.close()
    c.ctx.close()


def test_graph(hts):  # noqa: F811
    """Captured, and replayed over new inputs between eager calls."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = Case(hts, "bf16", 80, 2, 1, 2, 32, 32, starts=0.05)
        T, N, G, H, K, V = c.shape
        at = c.at
        ins = [at[n] for n in ("q", "k", "v", "a", "b", "A")]
        seq = dict(a_bias=at["a_bias"], starts=at["starts"], h_in=at["h_in"], **c.more)
        y, h, states = torch.empty(T, N, H, V, dtype=c.ty, device="cuda"), torch.empty(N, H, K, V, device="cuda"), torch.empty(hts.delta_rule_states(T, N, H, K, V), device="cuda")
        g = {n: torch.empty(s, dtype=c.ty, device="cuda") for n, s in (("dq", (T, N, G, K)), ("dk", (T, N, G, K)), ("dv", (T, N, H, V)), ("da", (T, N, H)), ("db", (T, N, H)))}
        g.update(dA=torch.empty(H, device="cuda"), da_bias=torch.empty(H, device="cuda"), dh_in=torch.empty(N, H, K, V, device="cuda"))

        def call():
            c.ctx.hts_delta_rule(*ins, y, h_out=h, states=states, **seq)
            c.ctx.hts_delta_rule_backward(*ins, at["dy"], states, dh_out=at["dh_out"], **g, **seq)
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for _ in range(3):
            for n in ("q", "k", "v", "a", "b", "dy"):
                at[n].copy_(torch.randn_like(at[n]))
            call()
            stream.synchronize()
            want = {n: x.clone() for n, x in {"y": y, "h": h, **g}.items()}
            for x in (y, h, *g.values()):
                x.fill_(9.0)
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(want[n], x) for n, x in {"y": y, "h": h, **g}.items())
        c.ctx.close()
