"""The experts' bf16 products and the adapters as they are called beside other work: recorded into graphs, on two streams, behind
an error that another call left, together in layers, and their gradients against differences."""
import ctypes

import numpy as np
import pytest
import torch

from rows_cases import BF16, F32, close, normals, offsets_of, small_ints

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def record(f):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f()
    return g


def random_ids(rows, adapters, seed):
    """Runs of rows of one adapter, or of none."""
    rng = np.random.default_rng(seed)
    ids = np.repeat(rng.integers(-1, adapters, rows), rng.integers(1, 40, rows))[:rows]
    return torch.from_numpy(ids.astype(np.int32)).cuda()


# (rows, columns, rank, adapters): one by one; tiles and parts of the rows with sums in memory
ADAPTERS = [(20, 96, 16, 3), (4096, 1100, 24, 4), (2500, 1030, 33, 9)]


def adapter_calls(so, rows, cols, rank, n, seed, workspaces=False):
    """The five calls of a layer's forward and backward pass on tensors of their own: (static inputs, run, outputs)."""
    x, dy = normals((rows, cols), seed), normals((rows, cols), seed + 1)
    a, b = normals((n, rank, cols), seed + 2, 0.1), normals((n, cols, rank), seed + 3, 0.1)
    scales = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    ids = random_ids(rows, n, seed)
    v, u = (torch.full((rows, rank), 7.0, device="cuda") for _ in range(2))
    y, dx = (torch.full((rows, cols), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    da, db = torch.full((n, rank, cols), 7.0, device="cuda"), torch.full((n, cols, rank), 7.0, device="cuda")
    memory = lambda size: torch.empty(max(size, 16), dtype=torch.uint8, device="cuda") if workspaces else None  # noqa: E731
    wd, ww = (memory(f(rows, cols, rank, n)) for f in (so.sfc_lora_down_ws_size, so.sfc_lora_wgrad_ws_size))

    def run():
        so.sfc_lora_down(x, a, ids, v, scales, workspace=wd)
        so.sfc_lora_up(v, b, ids, y, base=dy)
        so.sfc_lora_down(dy, b, ids, u, scales, layout=so.SFC_B_KN, workspace=wd)
        so.sfc_lora_up(u, a, ids, dx, layout=so.SFC_B_KN)
        so.sfc_lora_wgrad(x, u, ids, da, layout=so.SFC_B_KN, workspace=ww)
        so.sfc_lora_wgrad(dy, v, ids, db, workspace=ww)
    return (x, dy, ids), run, (v, y, u, dx, da, db)


@pytest.mark.parametrize("shape", ADAPTERS)
def test_adapters_in_a_graph(so, shape):
    """Replays with new contents, eager calls of the same sizes between them."""
    inputs, run, out = adapter_calls(so, *shape, 1)
    others = [adapter_calls(so, *shape, seed) for seed in (11, 21)]
    run()
    graph = record(run)
    batches = [[t.clone() for t in o[0]] for o in others]
    want = []
    for batch in batches:
        for t, s in zip(inputs, batch):
            t.copy_(s)
        run()
        want.append([t.clone() for t in out])
    for i in (1, 0, 0, 1):
        for t, s in zip(inputs, batches[i]):
            t.copy_(s)
        for t in out:
            t.fill_(5)
        graph.replay()
        others[i][1]()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[i]))


@pytest.mark.parametrize("shape", ADAPTERS)
def test_graphs_with_workspaces_replayed_at_once(so, shape):
    """Recorded on one stream, replayed on two."""
    calls = [adapter_calls(so, *shape, 31 + 10 * i, workspaces=True) for i in range(2)]
    want = []
    for _, run, out in calls:
        run()
        want.append([t.clone() for t in out])
    graphs = [record(run) for _, run, _ in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for _, _, out in calls:
            for t in out:
                t.fill_(3)
        torch.cuda.synchronize()
        for _ in range(10):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for (_, _, out), w in zip(calls, want):
            assert all(torch.equal(p, q) for p, q in zip(out, w))


@pytest.mark.parametrize("shape", ADAPTERS)
def test_adapters_on_two_streams(so, shape):
    """Library memory is a stream's own; the caller's workspace changes no bits."""
    calls = [adapter_calls(so, *shape, 51 + 10 * i) for i in range(2)]
    want = []
    for i, (_, run, out) in enumerate(calls):
        run()
        want.append([t.clone() for t in out])
        _, again, other = adapter_calls(so, *shape, 51 + 10 * i, workspaces=True)
        again()
        assert all(torch.equal(p, q) for p, q in zip(out, other))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for (_, run, _), stream in zip(calls, streams):
            with torch.cuda.stream(stream):
                run()
    torch.cuda.synchronize()
    for (_, _, out), w in zip(calls, want):
        assert all(torch.equal(p, q) for p, q in zip(out, w))


def test_a_workspace_that_is_too_small_is_refused(so):
    rows, cols, rank, n = ADAPTERS[1]
    (x, dy, ids), run, (v, y, u, dx, da, db) = adapter_calls(so, rows, cols, rank, n, 3)
    a = normals((n, rank, cols), 4)
    for size, call in ((so.sfc_lora_down_ws_size(rows, cols, rank, n), lambda ws: so.sfc_lora_down(x, a, ids, v, workspace=ws)),
                       (so.sfc_lora_wgrad_ws_size(rows, cols, rank, n), lambda ws: so.sfc_lora_wgrad(x, v, ids, db, workspace=ws))):
        assert size > 0
        ws = torch.full((size + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        v.zero_(), db.zero_()
        for short in (size - 1, 0):
            with pytest.raises(so.SfcError, match="workspace"):
                call(ws[:short])
        torch.cuda.synchronize()
        assert (ws == 0x5A).all() and not v.any() and not db.any()
        call(ws[:size])
        torch.cuda.synchronize()
        assert (ws[size:] == 0x5A).all()


def expert_calls(so, counts, N, K, seed):
    """Forward, gradient of the rows and of the weights for bf16 experts on tensors of their own."""
    rows, E = sum(counts), len(counts)
    x, w, dy = normals((rows, K), seed), normals((E, N, K), seed + 1, 0.1), normals((rows, N), seed + 2)
    offsets = offsets_of(counts)
    y, dx, dw = torch.zeros((rows, N), dtype=BF16, device="cuda"), torch.zeros((rows, K), device="cuda"), torch.zeros((E, N, K), device="cuda")

    def run():
        so.sfc_moe_gemm_ex(x, w, offsets, y)
        so.sfc_moe_gemm_ex(dy, w, offsets, dx, layout=so.SFC_B_KN)
        so.sfc_moe_wgrad_ex(dy, x, offsets, dw)
    return (x, w, dy, offsets), run, (y, dx, dw)


@pytest.mark.parametrize("counts,N,K", [([3, 0, 4], 200, 264), ([100, 300, 0, 56], 1290, 531), ([1500, 700], 2030, 1200)])
def test_experts_in_a_graph_and_on_two_streams(so, counts, N, K):
    """The recorded call is the first of its grid, so that its curve table is made there; segments change between replays."""
    (x, w, dy, offsets), run, out = expert_calls(so, counts, N, K, 1)
    graph = record(run)
    starts = [offsets.clone(), offsets_of(counts[::-1])]
    want = []
    for o in starts:
        offsets.copy_(o)
        run()
        want.append([t.clone() for t in out])
    for i in (1, 0, 1):
        offsets.copy_(starts[i])
        for t in out:
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[i]))
    calls = [expert_calls(so, counts, N, K, 40 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for (_, f, _), stream in zip(calls, streams):
        with torch.cuda.stream(stream):
            f()
    torch.cuda.synchronize()
    got = [[t.clone() for t in o] for _, _, o in calls]
    for (_, f, o), g in zip(calls, got):
        f()
        assert all(torch.equal(p, q) for p, q in zip(o, g))


def test_an_error_that_another_call_left_is_not_theirs(so):
    hip = so.lib                                     # (the library's own HIP runtime)
    hip.hipSetDevice.argtypes = [ctypes.c_int]
    for _, run, out in (adapter_calls(so, *ADAPTERS[0], 1), adapter_calls(so, 4095, 1100, 24, 4, 1), expert_calls(so, [3, 0, 4], 200, 264, 1),
                        expert_calls(so, [100, 300, 0, 57], 1310, 531, 1)):
        torch.cuda.synchronize()
        assert hip.hipSetDevice(1000) != 0
        try:
            run()
        finally:
            hip.hipGetLastError()                    # torch would report it as one of its own launches'
        got = [t.clone() for t in out]
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, got))


# ---- together ------------------------------------------------------------------------------------


@pytest.mark.parametrize("T", [1, 5, 300, 3000])
def test_a_layer_of_experts(so, T):
    """Sort, gather within the product, weighted sum; backwards to the tokens, the weights and the router's weights.  Whole numbers:
    every sum is exact."""
    k, E, K, N = 2, 8, 160, 224
    rows = so.sfc_moe_sort_rows(T * k, E, 1)
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.stack([torch.randperm(E, generator=g, device="cuda")[:k] for _ in range(T)]).to(I32)
    x, w, dy = small_ints((T, K), 1, most=4), small_ints((E, N, K), 2, most=4), small_ints((T, N), 3, most=4)
    weights = torch.randint(1, 4, (T, k), generator=g, device="cuda").float()
    new = lambda n: torch.empty(n, dtype=I32, device="cuda")  # noqa: E731
    offsets, order, pos = new(E + 1), new(rows), new(T * k)
    so.sfc_moe_sort(ids, offsets, order, pos)
    ys, y = torch.empty((rows, N), device="cuda"), torch.empty((T, N), device="cuda")
    so.sfc_moe_gemm_ex(x, w, offsets, ys, order=order, topk=k)
    so.sfc_moe_combine(ys, pos, y, weights=weights)
    wd = w.double()
    each = torch.stack([torch.stack([wd[int(e)] @ x[t].double() for e in ids[t]]) for t in range(T)])       # (T, k, N)
    assert torch.equal(y.double(), (each * weights[..., None]).sum(1))
    # the sum's gradient, in the sorted rows' type
    dys, dweights = torch.empty((rows, N), dtype=BF16, device="cuda"), torch.empty((T, k), device="cuda")
    so.sfc_moe_combine_grad(dy, ys.to(BF16), order, pos, weights, dys, dweights)
    dxs, dx, dw = torch.empty((rows, K), device="cuda"), torch.empty((T, K), device="cuda"), torch.empty((E, N, K), device="cuda")
    so.sfc_moe_gemm_ex(dys, w, offsets, dxs, layout=so.SFC_B_KN)
    so.sfc_moe_combine(dxs, pos, dx)
    xs = torch.empty((rows, K), dtype=BF16, device="cuda")
    so.sfc_moe_dispatch(x, order, xs, topk=k)
    so.sfc_moe_wgrad_ex(dys, xs, offsets, dw)
    want_dx, want_dw = torch.zeros_like(dx, dtype=torch.float64), torch.zeros_like(dw, dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            e, d = int(ids[t, j]), dy[t].double() * weights[t, j].double()
            want_dx[t] += d @ wd[e]
            want_dw[e] += d[:, None] * x[t].double()
    assert torch.equal(dx.double(), want_dx) and torch.equal(dw.double(), want_dw)


@pytest.mark.parametrize("rows", [1, 24, 3000])
def test_adapters_beside_a_shared_projection(so, rows):
    """Y = X W^T + the adapters' part, in place, and the gradients of X, A and B; whole numbers, exact."""
    from paper_2601_16294_amd import sfcgemm as sg
    K, N, rank, n = 320, 272, 40, 5
    x, w, dy = small_ints((rows, K), 1, most=2), small_ints((K, N), 2, most=2), small_ints((rows, N), 3, most=2)
    a, b = small_ints((n, rank, K), 4, most=2), small_ints((n, N, rank), 5, most=2)
    ids, scales = random_ids(rows, n, rows), torch.tensor([1.0, 2.0, 0.5, -1.0, 4.0], device="cuda")
    v, u = (torch.empty((rows, rank), device="cuda") for _ in range(2))
    y, dx = torch.empty((rows, N), device="cuda"), torch.empty((rows, K), device="cuda")
    sg.sfc_gemm_ex(x, w, y)
    so.sfc_lora_down(x, a, ids, v, scales)
    so.sfc_lora_up(v, b, ids, y, base=y)
    sg.sfc_gemm_ex(dy, w.t().contiguous(), dx)
    so.sfc_lora_down(dy, b, ids, u, scales, layout=so.SFC_B_KN)
    so.sfc_lora_up(u, a, ids, dx, base=dx, layout=so.SFC_B_KN)
    da, db = torch.empty((n, rank, K), device="cuda"), torch.empty((n, N, rank), device="cuda")
    so.sfc_lora_wgrad(x, u, ids, da, layout=so.SFC_B_KN)
    so.sfc_lora_wgrad(dy, v, ids, db)
    xd, dyd = x.double(), dy.double()
    want_y, want_dx = xd @ w.double(), dyd @ w.double().t()
    for i in range(n):
        t = torch.nonzero(ids == i)[:, 0]
        s, ad, bd = scales[i].double(), a[i].double(), b[i].double()
        want_y[t] += s * (xd[t] @ ad.t()) @ bd.t()
        want_dx[t] += s * (dyd[t] @ bd) @ ad
        # sums past 2^24 are rounded: magnitudes of what is added up bound them
        uu, vv = s * (dyd[t] @ bd), s * (xd[t] @ ad.t())
        assert close(da[i], uu.t() @ xd[t], uu.abs().t() @ xd[t].abs(), 3 * len(t) + 2, F32)
        assert close(db[i], dyd[t].t() @ vv, dyd[t].abs().t() @ vv.abs(), 3 * len(t) + 2, F32)
    assert torch.equal(y.double(), want_y) and torch.equal(dx.double(), want_dx)


def differences(loss, t, places, h):
    """Central differences of loss() (of a function of degree 2 at most in t: exact but for rounding) at elements of t."""
    out = []
    flat = t.view(-1)
    for i in places:
        keep = flat[i].clone()
        flat[i] = keep + h
        up = loss()
        flat[i] = keep - h
        down = loss()
        flat[i] = keep
        out.append((up - down) / (2 * h))
    return out


@pytest.mark.parametrize("rows", [12, 2600])
def test_gradients_of_adapters_against_differences(so, rows):
    """loss = sum of dY * Y with whole numbers: linear in every element, sums exact, so that a difference is the gradient."""
    K, N, rank, n = 80, 72, 16, 3
    x, dy = small_ints((rows, K), 1, most=1).contiguous(), small_ints((rows, N), 2, most=1).contiguous()
    a, b = small_ints((n, rank, K), 3, most=1).contiguous(), small_ints((n, N, rank), 4, most=1).contiguous()
    ids = random_ids(rows, n, 7)
    scales = torch.tensor([1.0, 2.0, 4.0], device="cuda")
    v, u = (torch.empty((rows, rank), device="cuda") for _ in range(2))
    y, dx = torch.empty((rows, N), device="cuda"), torch.empty((rows, K), device="cuda")

    def loss():
        so.sfc_lora_down(x, a, ids, v, scales)
        so.sfc_lora_up(v, b, ids, y)
        return float((y.double() * dy.double()).sum())

    loss()
    so.sfc_lora_down(dy, b, ids, u, scales, layout=so.SFC_B_KN)
    so.sfc_lora_up(u, a, ids, dx, layout=so.SFC_B_KN)
    da, db = torch.empty((n, rank, K), device="cuda"), torch.empty((n, N, rank), device="cuda")
    so.sfc_lora_wgrad(x, u, ids, da, layout=so.SFC_B_KN)
    so.sfc_lora_wgrad(dy, v, ids, db)
    rng = np.random.default_rng(rows)
    for t, grad in ((x, dx), (a, da), (b, db)):
        places = [int(i) for i in rng.integers(0, t.numel(), 12)]
        got = [float(grad.reshape(-1)[i]) for i in places]
        # (sums of up to rows * 2 * 4 * 80 < 2^24 whole numbers)
        assert differences(loss, t, places, 1.0) == got


@pytest.mark.parametrize("counts", [[3, 0, 5], [300, 200, 0, 70]])
def test_gradients_of_experts_against_differences(so, counts):
    K, N = 70, 90
    (x, w, dy, offsets), run, _ = expert_calls(so, counts, N, K, 1)
    rows, E = sum(counts), len(counts)
    x, w, dy = (small_ints(t.shape, 5 + i, most=3).contiguous() for i, t in enumerate((x, w, dy)))
    y, dx, dw = torch.empty((rows, N), device="cuda"), torch.empty((rows, K), device="cuda"), torch.empty((E, N, K), device="cuda")

    def loss():
        so.sfc_moe_gemm_ex(x, w, offsets, y)
        return float((y.double() * dy.double()).sum())

    so.sfc_moe_gemm_ex(dy, w, offsets, dx, layout=so.SFC_B_KN)
    so.sfc_moe_wgrad_ex(dy, x, offsets, dw)
    rng = np.random.default_rng(rows)
    for t, grad in ((x, dx), (w, dw)):
        places = [int(i) for i in rng.integers(0, t.numel(), 12)]
        assert differences(loss, t, places, 1.0) == [float(grad.reshape(-1)[i]) for i in places]


# ---- calls that the documents allow and that are rare --------------------------------------------


@pytest.mark.parametrize("rows,cols,rank,n", [(30, 77, 9, 3), (4096, 1100, 24, 4), (4096, 1100, 24, 1), (2500, 1031, 33, 9)])
def test_rows_of_no_adapter(so, rows, cols, rank, n):
    """None of a batch has one, whatever its V and its weights hold."""
    nan = lambda *s, dtype=BF16: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    ids = torch.full((rows,), -1, dtype=I32, device="cuda")
    ids[::3] = n
    x, v = normals((rows, cols), 1), torch.full((rows, rank), 9.0, device="cuda")
    so.sfc_lora_down(x, nan(n, rank, cols), ids, v, scales=nan(n, dtype=F32))
    assert not v.any()
    for dtype in (F32, BF16):
        base, y = normals((rows, cols), 2, dtype=dtype), nan(rows, cols, dtype=dtype)
        so.sfc_lora_up(nan(rows, rank, dtype=F32), nan(n, cols, rank), ids, y, base=base)
        assert torch.equal(y, base)
        so.sfc_lora_up(nan(rows, rank, dtype=F32), nan(n, cols, rank), ids, y)
        assert not y.any()
    g = nan(n, cols, rank, dtype=F32)
    so.sfc_lora_wgrad(nan(rows, cols), nan(rows, rank, dtype=F32), ids, g)
    assert not g.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,rank", [(30, 77, 9), (2500, 1031, 33), (5000, 514, 60), (2100, 1100, 40)])
@pytest.mark.parametrize("layout", [0, 1])
def test_up_in_place(so, rows, cols, rank, layout, dtype):
    """The same bits as into other memory, at odd elements too."""
    n = 3
    v, ids = normals((rows, rank), 1, dtype=F32), random_ids(rows, n, 5)
    b = normals((n, cols, rank) if layout == 0 else (n, rank, cols), 2)
    for pad, shift in ((0, 0), (1, 0), (0, 1), (3, 1), (6, 0)):
        base = normals((rows, cols), 3, ld_pad=pad, shift=shift, dtype=dtype)
        y = torch.empty((rows, cols), dtype=dtype, device="cuda")
        so.sfc_lora_up(v, b, ids, y, base=base, layout=layout)
        so.sfc_lora_up(v, b, ids, base, base=base, layout=layout)
        assert torch.equal(base, y)


def test_weights_that_all_share(so):
    """Experts and adapters of one matrix: a stride of 0 in the weights; gradients that would lie on each other are refused."""
    x, w, off = small_ints((40, 64), 1), small_ints((72, 64), 2), offsets_of([10, 0, 25, 5])
    y = torch.empty((40, 72), device="cuda")
    so.sfc_moe_gemm_ex(x, w.expand(4, 72, 64), off, y)
    assert torch.equal(y.double(), x.double() @ w.double().t())
    with pytest.raises(so.SfcError, match="overlap"):
        so.sfc_moe_wgrad_ex(y.to(BF16), x, off, torch.empty((72, 64), device="cuda").expand(4, 72, 64))
    ids, v = torch.arange(40, dtype=I32, device="cuda") % 3, torch.empty((40, 72), device="cuda")
    so.sfc_lora_down(x, w.expand(3, 72, 64), ids, v)
    assert torch.equal(v, y)
    with pytest.raises(so.SfcError, match="overlap"):
        so.sfc_lora_wgrad(x, v, ids, torch.empty((64, 72), device="cuda").expand(3, 64, 72))


@pytest.mark.parametrize("n,rows,cols,rank", [(1100, 3000, 40, 8), (33_000, 200, 16, 8), (1024, 20_000, 300, 5), (70_000, 50, 9, 3)])
def test_many_adapters(so, n, rows, cols, rank):
    """More than are counted in a workgroup, and more than a launch takes."""
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(-1, n + 1, (rows,), generator=g, device="cuda", dtype=I32)
    ids[:2], ids[2:4] = 0, n - 1
    x, a, b = small_ints((rows, cols), 1), small_ints((n, rank, cols), 2), small_ints((n, cols, rank), 3)
    v, y = torch.empty((rows, rank), device="cuda"), torch.empty((rows, cols), device="cuda")
    so.sfc_lora_down(x, a, ids, v)
    so.sfc_lora_up(v, b, ids, y)
    live = ((ids >= 0) & (ids < n))[:, None]
    at = ids.long().clamp(0, n - 1)
    want_v = torch.where(live, torch.bmm(a[at].float(), x.float()[:, :, None])[..., 0], 0.0)
    assert torch.equal(v, want_v)
    assert torch.equal(y, torch.where(live, torch.bmm(b[at].float(), want_v[:, :, None])[..., 0], 0.0))
    u = small_ints((rows, rank), 4).float()
    for layout in (0, 1):
        grad = torch.full((n, cols, rank) if layout == 0 else (n, rank, cols), 9.0, device="cuda")
        so.sfc_lora_wgrad(x, u, ids, grad, layout=layout)
        want = torch.zeros((n, cols, rank), device="cuda")
        want.index_add_(0, at, torch.where(live[..., None], x.float()[:, :, None] * u[:, None, :], 0.0))
        assert torch.equal(grad if layout == 0 else grad.transpose(1, 2), want)


def test_most_experts(so):
    counts = [(i * 7) % 5 for i in range(1024)]
    rows, N, K = sum(counts), 70, 130
    x, w, dy = small_ints((rows, K), 1), small_ints((1024, N, K), 2), small_ints((rows, N), 3)
    off, y, dw = offsets_of(counts), torch.empty((rows, N), device="cuda"), torch.empty((1024, N, K), device="cuda")
    so.sfc_moe_gemm_ex(x, w, off, y)
    so.sfc_moe_wgrad_ex(dy, x, off, dw)
    at = 0
    for e, n in enumerate(counts):
        s = slice(at, at + n)
        assert torch.equal(y[s].double(), x[s].double() @ w[e].double().t()) and torch.equal(dw[e].double(), dy[s].double().t() @ x[s].double())
        at += n


def test_one_expert_with_all_rows(so):
    """A batch of few rows on average whose router sends all of them to one of many experts."""
    E, N, K, rows = 64, 200, 264, 500
    x, w = small_ints((rows, K), 1), small_ints((E, N, K), 2)
    for e in (0, 17, E - 1):
        off = torch.tensor([0] * (e + 1) + [rows] * (E - e), dtype=I32, device="cuda")
        y = torch.empty((rows, N), device="cuda")
        so.sfc_moe_gemm_ex(x, w, off, y)
        assert torch.equal(y.double(), x.double() @ w[e].double().t())
