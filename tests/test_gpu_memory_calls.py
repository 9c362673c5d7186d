"""The recurrent core (memory.py): calls in orders and of sizes that a program makes and that nothing else here does."""
import pytest
import torch

from test_gpu_memory import small

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mem():
    import paper_2012_09849_amd.memory as m
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def test_fewer_sequences_than_the_most(mem):
    """A core for 17 sequences of 128 steps takes any smaller call: fewer sequences are worked on in more segments, whose workspace may be larger."""
    T, N = 128, 17
    core = small(mem, T=T, N=N, features=16, inner=1024, states=16)
    x, dy = torch.randn(T, N, 16, device="cuda"), torch.randn(T, N, 16, device="cuda")
    whole, state = torch.empty_like(x), mem.State(core, N)
    core.forward(x, whole, state)
    for n in (16, 3, 1):
        part, y, dx = x[:, :n].contiguous(), torch.empty(T, n, 16, device="cuda"), torch.empty(T, n, 16, device="cuda")
        core.forward(part, y, mem.State(core, n), train=True)
        core.backward(dy[:, :n].contiguous(), dx)
        torch.cuda.synchronize()
        # the order of sums, of the 128 steps' states, the 1024 channels and the projections of at most 1024 terms: 2^-24 for each on the way
        assert float((y - whole[:, :n]).abs().max()) <= 1500 * 2.0 ** -24 * float(whole.abs().max())
        assert bool(torch.isfinite(dx).all())
    core.close()


def test_a_step_ends_what_a_training_call_kept(mem):
    from paper_2012_09849_amd import HtsError
    core = small(mem, T=4, N=3)
    x, state = torch.randn(4, 3, 24, device="cuda"), mem.State(core, 3)
    core.forward(x, torch.empty_like(x), state, train=True)
    core.step(x[0], torch.empty(3, 24, device="cuda"), state)
    with pytest.raises(HtsError, match="backward"):
        core.backward(x, torch.empty_like(x))
    core.close()


def test_rows_within_a_wider_array_and_rows_that_are_not(mem):
    """Rows at one distance are taken in their place; others are refused, never copied."""
    from paper_2012_09849_amd import HtsError
    T, N, F = 4, 3, 24
    core = small(mem, T=T, N=N)
    x = torch.randn(T, N, F, device="cuda")
    y, wide = torch.empty_like(x), torch.zeros(T, N, F + 5, device="cuda")
    core.forward(x, y, mem.State(core, N))
    spread = torch.zeros(T, N, F + 3, device="cuda")
    spread[..., :F] = x
    core.forward(spread[..., :F], wide[..., 2:2 + F], mem.State(core, N))
    torch.cuda.synchronize()
    assert torch.equal(wide[..., 2:2 + F], y) and bool((wide[..., :2] == 0).all()) and bool((wide[..., 2 + F:] == 0).all())
    turned = torch.empty(N, T, F, device="cuda").transpose(0, 1)
    for a, b in ((turned, y), (x, turned), (x, y[:2]), (x, y.bfloat16())):
        with pytest.raises(HtsError):
            core.forward(a, b, mem.State(core, N))
    core.close()


def test_another_stream(mem):
    """A core on a stream of its own, made and initialised while the current stream is busy."""
    x = torch.randn(6, 5, 24, device="cuda")
    core = small(mem, T=6, N=5)
    want = torch.empty_like(x)
    core.forward(x, want, mem.State(core, 5))
    torch.cuda.synchronize()
    stream, busy = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    for _ in range(20):
        busy = busy @ busy * 1e-2
    other = mem.MemoryCore(24, 40, 8, 4, 6, core.precision, 6, 5, stream=stream)
    other.init_params(3)
    got = torch.empty_like(x)
    stream.wait_stream(torch.cuda.current_stream())
    other.forward(x, got, mem.State(other, 5))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    core.close()
    other.close()
