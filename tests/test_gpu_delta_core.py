"""The block around the gated delta rule (memory.DeltaCore): layer norm, products, convolution, rule and AdamW together, as a learner and an actor use them."""
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
    core = mem.DeltaCore(**{**dict(features=24, heads=4, groups=2, keys=8, values=12, width=4), **kw}, precision=PRECISION_BF16 if bf16 else PRECISION_FP32, max_steps=T, max_rows=N)
    core.init_params(3)
    return core


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("T", [9, 70])
def test_a_storage_in_one_call_and_step_by_step(mem, bf16, T):
    """In binary32 the two differ by the order of sums: 2^-24 for each of the 300 or so terms and roundings on a value's way (with chunks of 64 steps: of the substitution
    for each of them too, 8 sqrt(70 (64 x 64)) = 4300), of values of its size.  In bfloat16 the same operands are rounded the same way, but for those where that
    order decides: half a step (2^-8) of a few intermediate values."""
    N = 5
    core = small(mem, bf16, T=T)
    x = torch.randn(T, N, 24, device="cuda").to(core.dtype)
    starts = (torch.rand(T, N, device="cuda") < 0.15).to(torch.uint8)
    y, a, b = torch.empty_like(x), core.new_state(N), core.new_state(N)
    core.forward(x, y, a, starts=starts)
    one = torch.empty(N, 24, dtype=core.dtype, device="cuda")
    allowed = 8 * 2.0 ** -8 if bf16 else (300 if T < 17 else 4300) * 2.0 ** -24
    for t in range(T):
        core.step(x[t], one, b, starts[t])
        assert float((one.float() - y[t].float()).abs().max()) <= allowed * float(y.float().abs().max())
    assert float((a.h - b.h).abs().max()) <= allowed * float(a.h.abs().max()) and float((a.conv - b.conv).abs().max()) <= allowed * float(a.conv.abs().max())
    core.close()


def test_gradients_are_the_differences(mem):
    """The loss along random directions, binary32 with a step of 1e-2 of the parameters' size: differences are off by the loss's own roundings over twice
    the step, about 2^-24 x 300 / 1e-2 = 1.8e-3 of its size, and by the square of the step."""
    T, N = 17, 4
    core = small(mem, T=T, N=N)
    x, dy = torch.randn(T, N, 24, device="cuda"), torch.randn(T, N, 24, device="cuda")
    starts = (torch.rand(T, N, device="cuda") < 0.1).to(torch.uint8)
    lengths = torch.tensor([T, 0, T - 3, 1], dtype=torch.int32, device="cuda")
    begun = core.new_state(N)
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
        assert abs((found[0] - found[1]) / 2 - want) <= 300 * 2.0 ** -24 * scale + 0.02 * abs(want), name
    way = torch.randn_like(x) * 1e-2
    up, down = value(x + way)[0], value(x - way)[0]
    want = float((dx.double() * way.double()).sum())
    assert abs((up - down) / 2 - want) <= 300 * 2.0 ** -24 * scale + 0.02 * abs(want)
    core.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer(mem, bf16, bits):
    """Every array moves, the matrices' copies with them; both kinds of cores."""
    import paper_2012_09849_amd as hts
    for core in (small(mem, bf16), mem.MemoryCore(features=24, inner=40, states=8, rank=6, precision=hts.PRECISION_BF16 if bf16 else hts.PRECISION_FP32, max_steps=24, max_rows=5)):
        core.init_params(1)
        opt = core.optimizer(bits=bits, weight_decay=0.1)
        x = torch.randn(24, 5, 24, device="cuda").to(core.dtype)
        y, dx, before = torch.empty_like(x), torch.empty_like(x), core.params.clone()
        for _ in range(2):
            core.forward(x, y, core.new_state(5), train=True)
            core.backward(y, dx)
            opt.hts_adamw_step(hts.AdamWHParams(lr=1e-2, max_grad_norm=1.0, seed=2))
        torch.cuda.synchronize()
        assert opt.step == 2 and bool(core.params.isfinite().all())
        for name, p in core.views(before).items():
            assert bool((p != core.p[name]).any()), name
            if name in core.matrices:
                assert torch.equal(core.m[name], core.p[name].to(core.dtype)), name
        opt.close()
        core.close()


def test_refusals(mem):
    import paper_2012_09849_amd as hts
    core = small(mem, T=4, N=3)
    x = torch.randn(4, 3, 24, device="cuda")
    y, state = torch.empty_like(x), core.new_state(3)
    with pytest.raises(hts.HtsError, match="at most"):
        core.forward(torch.randn(5, 3, 24, device="cuda"), torch.empty(5, 3, 24, device="cuda"), state)
    with pytest.raises(hts.HtsError, match="no forward"):
        core.backward(y, x)
    with pytest.raises(hts.HtsError, match="shares memory"):
        core.forward(x, x, state, train=True)
    core.forward(x, y, state, train=True)
    with pytest.raises(hts.HtsError, match="shares memory"):
        core.backward(y, x)
    core.step(x[0], y[0], state)
    with pytest.raises(hts.HtsError, match="no forward"):       # what was kept has been overwritten
        core.backward(y, torch.empty_like(x))
    core.close()


def test_blocks_in_a_stack(mem):
    """Two blocks, one's output the other's input and its gradient the other's: the second one's gradient of its input is the first one's of its output."""
    T, N = 20, 3
    first, second = small(mem, T=T, N=N), small(mem, T=T, N=N)
    second.init_params(8)
    x, dy = torch.randn(T, N, 24, device="cuda"), torch.randn(T, N, 24, device="cuda")

    def value(x):
        mid, y = torch.empty_like(x), torch.empty_like(x)
        first.forward(x, mid, first.new_state(N), train=True)
        second.forward(mid, y, second.new_state(N), train=True)
        return mid, float((y.double() * dy.double()).sum()), float((y.double() * dy.double()).abs().sum())
    _, _, scale = value(x)
    dmid, dx = torch.empty_like(x), torch.empty_like(x)
    second.backward(dy, dmid)
    first.backward(dmid, dx)
    way = torch.randn_like(x) * 1e-2
    kept = dx.clone()
    up, down = value(x + way)[1], value(x - way)[1]
    want = float((kept.double() * way.double()).sum())
    assert abs((up - down) / 2 - want) <= 600 * 2.0 ** -24 * scale + 0.02 * abs(want)
    first.close()
    second.close()


@pytest.mark.parametrize("bits", [0, 32, 8])
def test_example_runs(mem, bits):
    """On streams of the cores' own, with both optimisers."""
    import paper_2012_09849_amd as hts
    stream = torch.cuda.Stream()
    core = mem.DeltaCore(features=32, heads=2, keys=16, values=16, precision=hts.PRECISION_BF16, max_steps=32, max_rows=16, stream=stream)
    core.init_params()
    opt = core.optimizer(bits=bits, weight_decay=0.01) if bits else None
    losses = mem.train_recall(core, 3, optimizer=opt)
    assert len(losses) == 3 and all(0 < v < 100 for v in losses)
    if opt:
        opt.close()
    core.close()
