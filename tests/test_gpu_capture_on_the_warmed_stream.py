"""Graphs recorded on the stream that ran the same call once before: products whose curve tables that stream made."""
import pytest
import torch

from rows_cases import BF16, offsets_of, small_ints

pytestmark = pytest.mark.gpu


def gemm(i, sg, so):
    x, w, y = small_ints((330 + i, 264), 1), small_ints((264, 2000 + 8 * i), 2), torch.empty((330 + i, 2000 + 8 * i), device="cuda")
    return lambda: sg.sfc_gemm_ex(x, w, y, tile="128x128"), y, lambda: x.double() @ w.double()


def experts_gradient(i, sg, so):
    counts = [70, 0, 130 + i]
    a, b = small_ints((sum(counts), 900 + 128 * i), 3), small_ints((sum(counts), 3000), 4)
    off, g = offsets_of(counts), torch.empty((3, 900 + 128 * i, 3000), device="cuda")

    def want():
        return torch.stack([a[s].double().t() @ b[s].double() for s in (slice(0, 70), slice(70, 70), slice(70, None))])
    return lambda: so.sfc_moe_wgrad_ex(a, b, off, g), g, want


@pytest.mark.parametrize("make", [gemm, experts_gradient])
def test_recorded_after_one_call_on_the_same_stream(make):
    from paper_2601_16294_amd import sfcgemm as sg
    from paper_2601_16294_amd import sfcops as so
    for i in range(2):
        run, out, want = make(i, sg, so)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream, capture_error_mode=("relaxed", "global")[i]):    # (torch waits for the device first)
            run()
        right = want()
        assert torch.equal(out.double(), right)
        for _ in range(3):
            out.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.double(), right)
        run()
        torch.cuda.synchronize()
        assert torch.equal(out.double(), right)
