"""What the kernels of the built library need: registers that are spilled to memory cost more than what they save.  No GPU is
needed."""
import pytest

import kernel_notes
from rows_cases import EXPERTS
from test_rows_routes import exe, launches, one  # noqa: F401


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


def test_few_rows_of_experts_have_no_kernel_that_no_call_takes(kernels, exe):
    """What is compiled of the kernel that streams the experts' weights, against what the host layer asks for."""
    asked = set()
    for rows in (1, 2, 8, 16, 17, 32, 33, 64, 65, 512):
        for experts in (1, 2, 8, 64, 1024):
            for K in (4096, 4095):
                for name, e in launches(one(exe, "experts", rows, 512, K, experts)):
                    if name == "rows":
                        asked.add((e["fm"], e["fn"]))
    compiled = {tuple(int(i) for i in n[n.index("<") + 1:].split(", ")[:2]) for n in kernels if n.startswith("moe_rows_kernel<")}
    assert compiled == asked


def test_gathered_bf16_products_of_the_gpu_tests_reach_every_block(kernels, exe):
    """What test_gpu_moe_bf16_order.py runs (two rows behind the last segment), past the caches or not aside."""
    reached = set()
    for c, N, K in EXPERTS:
        if sum(c):
            for layout in (0, 1):
                for pad in (0, 5):
                    (name, e), = launches(one(exe, "experts", sum(c) + 2, N, K, len(c), layout, 1, pad=pad))
                    reached.add((e["b"], layout) if name == "tile" else ("rows", layout))
    assert reached >= {(b, layout) for b in (64, 128, 256) for layout in (0, 1)} | {("rows", 0)}
