"""The recurrent core (memory.py): the operators together, as a learner and an actor use them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mem():
    import paper_2012_09849_amd.memory as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def small(mem, bf16=False, T=24, N=5, **kw):
    from paper_2012_09849_amd import PRECISION_BF16, PRECISION_FP32
    core = mem.MemoryCore(**{**dict(features=24, inner=40, states=8, rank=6, width=4), **kw}, precision=PRECISION_BF16 if bf16 else PRECISION_FP32, max_steps=T, max_rows=N)
    core.init_params(3)
    return core


@pytest.mark.parametrize("bf16", [False, True])
def test_a_storage_in_one_call_and_step_by_step(mem, bf16):
    """In binary32 the two differ by the order of sums: 2^-24 for each of the 200 or so terms and roundings on a value's way, of values of its size.  In
    bfloat16 the same operands are rounded the same way, but for those where that order decides: half a step (2^-8) of a few intermediate values."""
    T, N = 24, 5
    core = small(mem, bf16)
    x = torch.randn(T, N, 24, device="cuda").to(core.dtype)
    starts = (torch.rand(T, N, device="cuda") < 0.15).to(torch.uint8)
    y, a, b = torch.empty_like(x), mem.State(core, N), mem.State(core, N)
    core.forward(x, y, a, starts=starts)
    one = torch.empty(N, 24, dtype=core.dtype, device="cuda")
    allowed = 8 * 2.0 ** -8 if bf16 else 200 * 2.0 ** -24
    for t in range(T):
        core.step(x[t], one, b, starts[t])
        assert float((one.float() - y[t].float()).abs().max()) <= allowed * float(y.float().abs().max())
    assert float((a.h - b.h).abs().max()) <= allowed * float(a.h.abs().max()) and float((a.conv - b.conv).abs().max()) <= allowed * float(a.conv.abs().max())
    core.close()


def test_gradients_are_the_differences(mem):
    """The loss along random directions, binary32 with a step of 1e-2 of the parameters' size: differences are off by the loss's own roundings over twice
    the step, about 2^-24 x 200 / 1e-2 = 1.2e-3 of its size, and by the square of the step."""
    T, N = 17, 4
    core = small(mem, T=T, N=N)
    x, dy = torch.randn(T, N, 24, device="cuda"), torch.randn(T, N, 24, device="cuda")
    starts = (torch.rand(T, N, device="cuda") < 0.1).to(torch.uint8)
    lengths = torch.tensor([T, 0, T - 3, 1], dtype=torch.int32, device="cuda")
    begun = mem.State(core, N)
    begun.h.normal_()
    begun.conv.normal_()
    live = (torch.arange(T, device="cuda")[:, None] < lengths)[:, :, None]

    def value(x):
        y = torch.empty_like(x)
        core.forward(x.contiguous(), y, begun.clone(), starts=starts, lengths=lengths, train=True)
        return float((y.double() * dy.double() * live).sum()), float((y.double() * dy.double() * live).abs().sum())
    scale = value(x)[1]
    masked = (dy * live).contiguous()
    dx = torch.empty_like(x)
    core.backward(masked, dx)
    grads, kept = core.grads.clone(), core.params.clone()
    for name, view in core.views(grads).items():
        way = torch.randn_like(view) * 1e-2 * max(float(core.p[name].abs().max()), 0.1) / view.numel() ** 0.5
        found = []
        for sign in (1, -1):
            core.params.copy_(kept)
            core.p[name].add_(sign * way)
            found.append(value(x)[0])
        core.params.copy_(kept)
        want = float((view.double() * way.double()).sum())
        assert abs((found[0] - found[1]) / 2 - want) <= 200 * 2.0 ** -24 * scale + 0.02 * abs(want), name
    way = torch.randn_like(x) * 1e-2
    up, down = value(x + way)[0], value(x - way)[0]
    want = float((dx.double() * way.double()).sum())
    assert abs((up - down) / 2 - want) <= 200 * 2.0 ** -24 * scale + 0.02 * abs(want)
    core.close()


@pytest.mark.parametrize("bf16", [False, True])
def test_it_learns_to_recall(mem, bf16):
    core = small(mem, bf16, T=32, N=16, features=32, inner=64, states=16, rank=8)
    losses = mem.train_recall(core, 120, T=32, N=16)
    assert np.isfinite(losses).all() and np.mean(losses[-10:]) < 0.5 * np.mean(losses[:3]) and losses[0] > 0.5
    core.close()


def test_steps_in_a_graph(mem):
    """An actor's step recorded once and replayed, with eager work between: every replay moves the state on as the eager call does."""
    core = small(mem, T=1, N=8)
    x, starts = torch.randn(6, 8, 24, device="cuda"), torch.zeros(8, dtype=torch.uint8, device="cuda")
    want, ref = [], mem.State(core, 8)
    for t in range(6):
        y = torch.empty(8, 24, device="cuda")
        core.step(x[t], y, ref, starts)
        want.append(y)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    from paper_2012_09849_amd import PRECISION_FP32
    other = mem.MemoryCore(24, 40, 8, 4, 6, PRECISION_FP32, 1, 8, stream=stream)
    other.params.copy_(core.params)
    state, xin, yout = mem.State(other, 8), torch.zeros(8, 24, device="cuda"), torch.zeros(8, 24, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        other.step(xin, yout, state, starts)
    torch.cuda.synchronize()
    for t in range(6):
        xin.copy_(x[t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yout, want[t]), t
        torch.randn(1000, device="cuda").sum().item()
    assert torch.equal(state.h, ref.h) and torch.equal(state.conv, ref.conv)
    core.close()
    other.close()


def test_what_it_refuses(mem):
    from paper_2012_09849_amd import HtsError
    core = small(mem, T=4, N=3)
    state = mem.State(core, 3)
    for shape in ((5, 3, 24), (4, 4, 24), (4, 3, 23)):
        x = torch.zeros(*shape, device="cuda")
        with pytest.raises(HtsError):
            core.forward(x, torch.empty_like(x), state)
    x = torch.zeros(4, 3, 24, device="cuda")
    core.forward(x, torch.empty_like(x), state)
    with pytest.raises(HtsError):
        core.backward(x, torch.empty_like(x))
    with pytest.raises(HtsError):
        core.ctx.hts_linear(x[0], core.m["in.w"], torch.empty(3, 7, device="cuda"))
    with pytest.raises(HtsError):
        core.ctx.hts_linear(x[0].t(), core.m["in.w"].t(), torch.empty(24, 3, device="cuda"))
    core.close()
