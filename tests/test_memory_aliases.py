"""The recurrent core (memory.py): arrays that a training call reads again and that another one would overwrite are refused."""
import pytest
import torch


def test_rows_that_share_memory():
    """Against the entries written down one by one, for rows within a wider array, of any distance."""
    from paper_2012_09849_amd.memory import _meet
    g = torch.Generator().manual_seed(1)
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (), generator=g))  # noqa: E731
    whole, seen = torch.zeros(600), {True: 0, False: 0}
    for k in range(3000):
        ld, to = pick(0, 20), pick(0, 20)
        a, b = (whole.as_strided((pick(1, 8), pick(1, 12)), (d, 1), pick(0, 200)) for d in (ld, ld if k % 3 == 0 else to))
        whole.zero_()
        a.fill_(1)
        want = bool((b != 0).any())
        assert _meet(a, b) == want and _meet(b, a) == want, (a.shape, a.stride(), a.storage_offset(), b.shape, b.stride(), b.storage_offset())
        seen[want] += 1
    assert min(seen.values()) > 300


@pytest.mark.gpu
def test_what_a_training_call_refuses():
    import paper_2012_09849_amd as hts
    from paper_2012_09849_amd import memory
    from test_gpu_memory import small
    T, N, F = 4, 3, 24
    core = small(memory, T=T, N=N)
    x = torch.randn(T, N, F, device="cuda")
    y, state = torch.empty_like(x), memory.State(core, N)
    core.forward(x, y, state)
    place, again = x.clone(), memory.State(core, N)
    core.forward(place, place, again)                           # without a backward pass y may take x's place
    torch.cuda.synchronize()
    assert torch.equal(place, y) and torch.equal(again.h, state.h)
    wide = torch.zeros(T, N, 2 * F, device="cuda")
    wide[..., :F] = x
    for bad in (x, wide[..., F - 1:2 * F - 1]):
        before = memory.State(core, N)
        with pytest.raises(hts.HtsError, match="shares memory"):
            core.forward(x if bad is x else wide[..., :F], bad, before, train=True)
        assert bool((before.h == 0).all())
    dy = torch.randn(T, N, F, device="cuda")
    dx, beside = torch.empty_like(x), wide[..., F:]
    core.forward(wide[..., :F], beside, memory.State(core, N), train=True)             # between x's rows: nothing is shared
    assert torch.equal(beside, y)
    core.backward(dy, dx)
    grads = core.grads.clone()
    for bad in (dy, wide[..., 1:F + 1]):
        with pytest.raises(hts.HtsError, match="shares memory"):
            core.backward(dy, bad)
    core.backward(dy, beside)                                   # refused calls change nothing
    torch.cuda.synchronize()
    assert torch.equal(core.grads, grads) and torch.equal(beside, dx)
    core.close()
