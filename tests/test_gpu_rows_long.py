"""Experts' bf16 products and adapters on operands and results of more than 2^31 elements, more rows than a launch takes and
columns past 2^20: whole numbers, exact, compared where offsets pass 32 bits and at the ends."""
import pytest
import torch

from rows_cases import BF16, F32

pytestmark = pytest.mark.gpu
I32 = torch.int32
ROWS, COLS = 600_001, 4100                   # 2.46e9 elements
CROSS = (1 << 31) // COLS                    # the row at element 2^31


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


@pytest.fixture(scope="module")
def big():
    """(ROWS, COLS) whole numbers -2 .. 2."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((ROWS, COLS), dtype=BF16, device="cuda")
    for i in range(0, ROWS, 100_000):
        part = x[i:i + 100_000]
        part.copy_(torch.randint(-2, 3, part.shape, generator=g, device="cuda", dtype=torch.int8))
    yield x
    del x, part
    torch.cuda.empty_cache()


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def ints(*shape, seed=2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(BF16)


def picked(rows):
    """Rows at the start, around element 2^31, at the end and all over."""
    return torch.cat([torch.arange(0, 70), torch.arange(CROSS - 70, CROSS + 70), torch.arange(rows - 70, rows),
                      torch.arange(0, rows, 997)]).cuda()


@pytest.mark.parametrize("layout", [0, 1])
def test_experts_of_long_batches(so, big, layout):
    N, starts = 40, [0, 100_000, 100_000, CROSS + 1000, ROWS - 1]
    E = len(starts) - 1
    w = ints(E, N, COLS) if layout == 0 else ints(E, COLS, N)
    c = torch.full((ROWS, N), 9.0, device="cuda")
    so.sfc_moe_gemm_ex(big, w, torch.tensor(starts, dtype=I32, device="cuda"), c, layout=layout)
    t = picked(ROWS - 1)
    e = torch.bucketize(t, torch.tensor(starts[1:], device="cuda"), right=True)
    for i in range(E):
        m = t[e == i]
        assert torch.equal(c[m].double(), big[m].double() @ (w[i].double().t() if layout == 0 else w[i].double()))
    assert not c[-1].any()


def test_experts_weight_gradient_of_long_batches(so, big):
    starts = [0, 64, CROSS - 100, CROSS + 100, ROWS - 300, ROWS]
    b = ints(ROWS, 24)
    g = torch.full((5, COLS, 24), 9.0, device="cuda")
    so.sfc_moe_wgrad_ex(big, b, torch.tensor(starts, dtype=I32, device="cuda"), g)
    for i in (0, 2, 4):
        s = slice(starts[i], starts[i + 1])
        assert torch.equal(g[i].double(), big[s].double().t() @ b[s].double())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_experts_with_a_long_result(so, dtype):
    rows, N = 40_003, 60_007
    a, w = ints(rows, 8), ints(2, N, 8, seed=3)
    c = torch.full((rows, N), 9.0, dtype=dtype, device="cuda")
    so.sfc_moe_gemm_ex(a, w, torch.tensor([0, 20_000, rows], dtype=I32, device="cuda"), c)
    for i in range(0, rows, 4000):
        for lo, hi, e in ((i, min(i + 4000, 20_000), 0), (max(i, 20_000), min(i + 4000, rows), 1)):
            if lo < hi:
                assert torch.equal(c[lo:hi], (a[lo:hi].float() @ w[e].float().t()).to(dtype))


def test_experts_with_long_weights(so):
    E, N, K = 1000, 1200, 2048                # 2.46e9 elements
    w = torch.empty((E, N, K), dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    for e in range(0, E, 50):
        w[e:e + 50].copy_(torch.randint(-2, 3, (50, N, K), generator=g, device="cuda", dtype=torch.int8))
    a, c = ints(E, K), torch.empty((E, N), device="cuda")
    so.sfc_moe_gemm_ex(a, w, torch.arange(E + 1, dtype=I32, device="cuda"), c)
    for e in (0, 1, 872, 873, 874, 875, E - 2, E - 1):
        assert torch.equal(c[e].double(), w[e].double() @ a[e].double())
    out = torch.full((E, N, K), 9.0, dtype=BF16, device="cuda")
    so.sfc_moe_wgrad_ex(ints(E, N, seed=6), a, torch.arange(E + 1, dtype=I32, device="cuda"), out)
    d = ints(E, N, seed=6)
    for e in (0, 873, 874, E - 1):
        assert torch.equal(out[e].float(), d[e].float()[:, None] * a[e].float())


@pytest.mark.parametrize("layout", [0, 1])
def test_adapters_of_long_batches(so, big, layout):
    n, rank = 3, 8
    a = ints(n, rank, COLS) if layout == 0 else ints(n, COLS, rank)
    ids = (torch.arange(ROWS, device="cuda") // 1000 % (n + 1)).to(I32)
    v = torch.full((ROWS, rank), 9.0, device="cuda")
    so.sfc_lora_down(big, a, ids, v, layout=layout)
    t = picked(ROWS)
    for i in range(n + 1):
        m = t[ids[t] == i]
        want = torch.zeros((len(m), rank), dtype=torch.float64, device="cuda") if i == n else \
            big[m].double() @ (a[i].double().t() if layout == 0 else a[i].double())
        assert torch.equal(v[m].double(), want)
    vs = ints(ROWS, rank, seed=8).float()
    y = torch.full((ROWS, COLS), 9.0, dtype=BF16, device="cuda")
    other = 1 - layout                       # (the same weights as up's)
    so.sfc_lora_up(vs, a, ids, y, base=big, layout=other)
    for i in range(n + 1):
        m = t[ids[t] == i]
        part = 0 if i == n else vs[m].double() @ (a[i].double().t() if other == 0 else a[i].double())
        assert torch.equal(y[m], (big[m].double() + part).to(BF16))
    if layout == 0:
        ids = torch.full((ROWS,), -1, dtype=I32, device="cuda")
        ids[CROSS - 100:CROSS + 100], ids[-300:], ids[:5] = 1, 2, 2
        g = torch.full((n, COLS, rank), 9.0, device="cuda")
        so.sfc_lora_wgrad(big, vs, ids, g)
        for i in range(n):
            m = torch.nonzero(ids == i)[:, 0]
            assert torch.equal(g[i].double(), big[m].double().t() @ vs[m].double())


def test_more_rows_than_a_launch_takes(so):
    rows, cols, rank, n = (1 << 22) + 4999, 40, 16, 2
    x, a, b = ints(rows, cols), ints(n, rank, cols), ints(n, cols, rank, seed=3)
    ids = (torch.arange(rows, device="cuda") // 77 % (n + 1)).to(I32)
    v, y = torch.full((rows, rank), 9.0, device="cuda"), torch.full((rows, cols), 9.0, device="cuda")
    so.sfc_lora_down(x, a, ids, v)
    so.sfc_lora_up(v, b, ids, y, base=x.float())
    want_v, want_y = torch.zeros_like(v), x.float()
    for i in range(n):
        m = (ids == i)[:, None]
        want_v = torch.where(m, x.float() @ a[i].float().t(), want_v)
        want_y = torch.where(m, x.float() + want_v @ b[i].float().t(), want_y)
    assert torch.equal(v, want_v) and torch.equal(y, want_y)
    g, size = torch.full((n, cols, rank), 9.0, device="cuda"), x.double()
    so.sfc_lora_wgrad(x, v, ids, g)
    for i in range(n):
        vd = v.double() * (ids == i)[:, None]
        assert ((g[i].double() - size.t() @ vd).abs() <= 2.0 ** -23 * (3 * rows + 2) * (size.abs().t() @ vd.abs())).all()


@pytest.mark.parametrize("rows", [3, 300])
def test_columns_past_a_launch(so, rows):
    cols, rank, n = (1 << 20) + 2051, 8, 2
    v, b = ints(rows, rank).float(), ints(n, cols, rank, seed=3)
    ids = (torch.arange(rows, device="cuda") // 2 % (n + 1)).to(I32)
    base = ints(rows, cols, seed=4)
    for layout, w in ((0, b), (1, b.transpose(1, 2).contiguous())):
        y = torch.full((rows, cols), 9.0, dtype=BF16, device="cuda")
        so.sfc_lora_up(v, w, ids, y, base=base, layout=layout)
        for t in {0, 2, rows - 1}:
            i = int(ids[t])
            part = 0 if i == n else b[i].float() @ v[t]
            assert torch.equal(y[t], (base[t].float() + part).to(BF16))
        g = torch.full((n, cols, rank) if layout == 0 else (n, rank, cols), 9.0, device="cuda")
        so.sfc_lora_wgrad(base, v, ids, g, layout=layout)
        for i in range(n):
            m = torch.nonzero(ids == i)[:, 0]
            want = base[m].float().t() @ v[m]
            assert torch.equal(g[i] if layout == 0 else g[i].t(), want)
