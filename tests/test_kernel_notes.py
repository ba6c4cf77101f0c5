"""What the kernels of the built library need: registers that are spilled to memory cost more than what they save.  No GPU is
needed."""
import pytest

import kernel_notes


@pytest.fixture(scope="module")
def kernels():
    return kernel_notes.kernels()


def test_adapters_keep_their_values_in_registers(kernels):
    """Every kernel of the adapters, at each rank."""
    mine = {n: k for n, k in kernels.items() if n.startswith("lora_")}
    assert len(mine) > 60
    spilled = {n: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) for n, k in mine.items()
               if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}
    assert not spilled
