"""The recurrent core on a stream of its own while the caller's stream is busy: the same bits as on the caller's."""
import pytest
import torch

from test_gpu_memory import small

pytestmark = pytest.mark.gpu


def test_training_on_a_stream_of_its_own():
    import paper_2012_09849_amd.memory as mem
    core = small(mem, T=32, N=16)
    want = mem.train_recall(core, 6)
    params = core.params.clone()
    torch.cuda.synchronize()
    core.close()
    stream, busy = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    other = mem.MemoryCore(24, 40, 8, 4, 6, core.precision, 32, 16, stream=stream)
    other.init_params(3)
    for _ in range(20):
        busy = busy @ busy * 1e-2
    got = mem.train_recall(other, 6)
    after = other.params + 0                                    # on the caller's stream, which has waited
    torch.cuda.synchronize()
    assert got == want and torch.equal(after, params)
    other.close()
