"""What a core's optimizer refuses."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [0, 4, 16, 64])
def test_states_of_other_sizes(bits):
    """States have 32 or 8 bits: others are refused, not made in 32."""
    import paper_2012_09849_amd as hts
    from paper_2012_09849_amd import memory
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    for core in (memory.DeltaCore(features=16, heads=2, keys=8, values=8), memory.MemoryCore(features=16, inner=16, states=8, rank=4)):
        with pytest.raises(hts.HtsError, match="32 or 8"):
            core.optimizer(bits=bits)
        core.close()
