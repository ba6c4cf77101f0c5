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


def sort_outputs(E, rows, slots):
    new = lambda n: torch.full((n,), 7, dtype=torch.int32, device="cuda")
    return new(E + 1), new(rows), new(slots)


@pytest.mark.parametrize("slots,E", [(5000, 8), (9000, 1024), (600000, 70)])
def test_sort_on_two_streams_and_in_a_graph(so, slots, E):
    """Past 4096 slots the sort has counts in library memory: one per stream, another for graphs."""
    g = torch.Generator(device="cuda").manual_seed(slots)
    ids = [torch.randint(-1, E, (slots,), generator=g, device="cuda", dtype=torch.int32) for _ in range(2)]
    want, got = ([sort_outputs(E, slots + E * 31, slots) for _ in range(2)] for _ in range(2))
    for i in range(2):
        so.sfc_moe_sort(ids[i], *want[i], align=32)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for i in range(2):
            so.sfc_moe_sort(ids[i], *got[i], align=32, stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(got[i], want[i]))
    static, out, eager = ids[0].clone(), sort_outputs(E, slots + E * 31, slots), sort_outputs(E, slots + E * 31, slots)
    graph = record(lambda: so.sfc_moe_sort(static, *out, align=32))
    for i in (1, 0, 1):
        static.copy_(ids[i])
        for t in (*out, *eager):
            t.fill_(7)
        graph.replay()
        so.sfc_moe_sort(ids[1 - i], *eager, align=32)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i])) and all(torch.equal(a, b) for a, b in zip(eager, want[1 - i]))


# (grids of blocks that no other test has: their curve tables are made here)
def test_weight_gradients_on_two_streams_at_once(so):
    M, N = 1700, 2500
    starts = [0, 96, 96, 800, 1024]
    offsets = torch.tensor(starts, dtype=torch.int32, device="cuda")
    A, B = ([operand(n, 1024, s + i) for i in range(2)] for n, s in ((M, 3), (N, 13)))
    got = [torch.zeros((4, M, N), device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):                     # the second call finds the table queued on the other stream
        so.sfc_moe_wgrad_mx4_ex(*A[i][:2], *B[i][:2], offsets, got[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for e, (lo, hi) in enumerate(zip(starts[:-1], starts[1:])):
            assert torch.equal(got[i][e].double(), A[i][2][:, lo:hi] @ B[i][2][:, lo:hi].t())


@pytest.mark.parametrize("M,N", [(1830, 2420), (1950, 2300)])
def test_weight_gradients_in_a_graph(so, M, N):
    """The first call of a grid is a recorded one: the graph holds its curve table."""
    starts = [[0, 96, 96, 800, 1024], [0, 512, 544, 544, 992]]
    (A, As, a), (B, Bs, b) = operand(M, 1024, 5), operand(N, 1024, 6)
    offsets = torch.tensor(starts[0], dtype=torch.int32, device="cuda")
    out, eager = (torch.zeros((4, M, N), device="cuda") for _ in range(2))
    graph = record(lambda: so.sfc_moe_wgrad_mx4_ex(A, As, B, Bs, offsets, out))
    for i in (0, 1, 0):
        offsets.copy_(torch.tensor(starts[i], dtype=torch.int32))
        out.fill_(3)
        graph.replay()
        so.sfc_moe_wgrad_mx4_ex(A, As, B, Bs, offsets, eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        for e, (lo, hi) in enumerate(zip(starts[i][:-1], starts[i][1:])):
            assert torch.equal(out[e].double(), a[:, lo:hi] @ b[:, lo:hi].t())


@pytest.mark.parametrize("T", [5, 300, 3000])
def test_a_layer_of_experts_in_a_graph(so, T):
    """Sort, gather to 4 bits, the experts' product, the weighted sum and its gradient as one graph."""
    k, E, K, N = 2, 8, 160, 224
    rows = so.sfc_moe_sort_rows(T * k, E, 32)
    wq = so.mx4_empty(N, K, lead=(E,))
    for e in range(E):
        so.sfc_mx4_quant(inputs(N, K, BF16, 50 + e), wq[0][e], wq[1][e])
    g = torch.Generator(device="cuda").manual_seed(T)
    batches = [(inputs(T, K, BF16, i), torch.stack([torch.randperm(E, generator=g, device="cuda")[:k] for _ in range(T)]).int(),
                torch.rand((T, k), generator=g, device="cuda"), inputs(T, N, BF16, 9 + i)) for i in range(2)]

    def layer(x, ids, w, dy):
        offsets, order, pos = sort_outputs(E, rows, T * k)
        so.sfc_moe_sort(ids, offsets, order, pos, align=32)
        xq, ys, y = so.mx4_empty(rows, K), torch.empty((rows, N), dtype=BF16, device="cuda"), torch.empty((T, N), dtype=BF16, device="cuda")
        so.sfc_mx4_quant(x, *xq, order=order, topk=k)
        so.sfc_moe_gemm_mx4_ex(*xq, *wq, offsets, ys)
        so.sfc_moe_combine(ys, pos, y, weights=w)
        dys, dw, dt, xt = torch.empty_like(ys), torch.empty((T, k), device="cuda"), so.mx4_empty(N, rows), so.mx4_empty(K, rows)
        so.sfc_moe_combine_grad(dy, ys, order, pos, w, dys, dw)
        so.sfc_mx4_quant(dys, None, None, *dt)
        so.sfc_mx4_quant(x, None, None, *xt, order=order, topk=k)
        dwe = torch.empty((E, N, K), device="cuda")
        so.sfc_moe_wgrad_mx4_ex(*dt, *xt, offsets, dwe)
        return y, dys, dw, dwe

    want = [[t.clone() for t in layer(*b)] for b in batches]
    static = [t.clone() for t in batches[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(*static)
    for i in (1, 0, 1, 1):
        for a, b in zip(static, batches[i]):
            a.copy_(b)
        graph.replay()
        eager = layer(*batches[1 - i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i])) and all(torch.equal(a, b) for a, b in zip(eager, want[1 - i]))
