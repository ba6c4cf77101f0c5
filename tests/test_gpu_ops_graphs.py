"""4-bit and expert calls recorded into graphs and on two streams: replays, eager calls between them
and replays that overlap each other give the bits of eager calls."""
import pytest
import torch

from test_gpu_mx4 import BF16, inputs, operand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def record(f):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):            # one capture stream for all of them
        f()
    return g


@pytest.mark.parametrize("entry", ["linear", "gemm"])
def test_graphs_with_workspaces_replayed_at_once(so, entry):
    """Two graphs that were recorded on one stream, replayed on two: each has its own codes and copies."""
    M, N, K = 300, 130, 8192
    W, Ws, _ = operand(N, K, 4)
    x = [inputs(M, K, BF16, i) for i in range(2)]
    q = [so.mx4_empty(M, K) for _ in range(2)]
    want, got = ([torch.empty((M, N), device="cuda") for _ in range(2)] for _ in range(2))
    n = so.sfc_mx4_linear_ws_size(M, N, K) if entry == "linear" else so.sfc_gemm_mx4_ws_size(M, N, K)
    assert n > 0
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(i, y, **kw):
        if entry == "linear":
            so.sfc_mx4_linear(x[i], W, Ws, y, **kw)
        else:
            so.sfc_gemm_mx4_ex(*q[i], W, Ws, y, **kw)

    for i in range(2):
        so.sfc_mx4_quant(x[i], *q[i])
        call(i, want[i])
    torch.cuda.synchronize()
    graphs = [record(lambda i=i: call(i, got[i], workspace=ws[i])) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for y in got:
            y.fill_(3)
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (16, 100, 4128), (40, 100, 128), (300, 130, 8192), (500, 520, 100)])
def test_a_workspace_changes_no_bits(so, M, N, K):
    W, Ws, _ = operand(N, -(-K // 32) * 32, 4)
    x = inputs(M, K, BF16, 1)
    for dtype in (torch.float32, BF16):
        want, got = torch.empty((M, N), dtype=dtype, device="cuda"), torch.empty((M, N), dtype=dtype, device="cuda")
        so.sfc_mx4_linear(x, W, Ws, want)
        n = so.sfc_mx4_linear_ws_size(M, N, K, dtype)
        ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        so.sfc_mx4_linear(x, W, Ws, got, workspace=ws[:n])
        assert torch.equal(got, want) and (ws[n:] == 0x5A).all()
        if n:
            with pytest.raises(so.SfcError, match="workspace"):
                so.sfc_mx4_linear(x, W, Ws, got, workspace=ws[:n - 1])
            with pytest.raises(so.SfcError, match="workspace"):
                so.sfc_mx4_linear(x, W, Ws, got, workspace=ws[:0])
