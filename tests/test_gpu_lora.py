"""Low-rank adapters on the GPU: down, up, their gradients and the weight gradients, against 64 bits.

Whole numbers whose sums fit 24 bits (and V of 16 bits) give exact fp32 results and bf16 results that are
their rounding, bit for bit; memory around the operands is NaN.  Normal values: bf16 products of K terms are
within (K + 1) * 2^-23 of the sum of magnitudes with the scale; V's products as well, with 2^-16 more where V is taken to 16
bits (bf16 Y); bf16 output adds 2^-8 of the result."""
import numpy as np
import pytest
import torch

from rows_cases import BF16, F32, close, framed, normals, small_ints, untouched_outside

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def make_ids(rows, adapters, seed, kind):
    """Rows that each have an adapter of their own, runs of rows, or one adapter; some with none."""
    rng = np.random.default_rng(seed)
    if kind == "rows":
        ids = rng.integers(-1, adapters + 1, rows)
    elif kind == "runs":
        ids = np.repeat(rng.integers(-1, adapters, rows), rng.integers(1, 50, rows))[:rows]
    else:
        ids = np.full(rows, adapters - 1)
    ids[rng.random(rows) < 0.05] = rng.choice([-1, -(1 << 31), adapters, (1 << 31) - 1])
    return torch.from_numpy(ids.astype(np.int32)).cuda()


def weights_of(w, ids):
    """(rows of each adapter, its weights)."""
    for a in range(w.shape[0]):
        yield torch.nonzero(ids == a)[:, 0], w[a].double()


def down(x, a, ids, scales, nk):
    v = torch.zeros((x.shape[0], a.shape[1 if nk else 2]), dtype=torch.float64, device="cuda")
    for i, (rows, w) in enumerate(weights_of(a, ids)):
        v[rows] = x[rows].double() @ (w.t() if nk else w) * (1.0 if scales is None else scales[i].double())
    return v


def up(v, b, ids, base, nk):
    y = base.double().clone()
    for rows, w in weights_of(b, ids):
        y[rows] += v[rows].double() @ (w.t() if nk else w)
    return y


def same(got, want):
    return torch.equal(got, want.float().to(got.dtype))


# (rows, columns, rank, adapters)
SHAPES = [(1, 1, 1, 1), (1, 4096, 16, 3), (5, 33, 7, 2), (16, 64, 16, 16), (32, 1000, 16, 8), (17, 130, 33, 4), (100, 70, 64, 1),
          (64, 65, 12, 5), (333, 257, 100, 3), (70, 515, 128, 2), (40, 96, 256, 3), (1000, 300, 8, 6), (2049, 640, 24, 9)]
# (too large to be taken row by row)
TILES = [(5000, 1030, 16, 5), (2500, 1030, 31, 9), (2100, 1100, 40, 2), (1300, 1000, 64, 3), (1500, 515, 100, 2), (1000, 600, 128, 3),
         (600, 520, 256, 4), (9700, 1030, 8, 6), (20000, 64, 64, 3), (8000, 800, 12, 3), (250, 2200, 256, 3)]
SHAPES += TILES


@pytest.mark.parametrize("rows,cols,rank,adapters", SHAPES)
@pytest.mark.parametrize("kind", ["rows", "runs", "one"])
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_down(so, rows, cols, rank, adapters, kind, nk, pad, shift):
    ids = make_ids(rows, adapters, rows + rank, kind)
    x = small_ints((rows, cols), 1, pad, shift)
    a = small_ints((adapters, rank, cols) if nk else (adapters, cols, rank), 2, pad, shift, gap=3)
    scales = torch.exp2(torch.arange(adapters, device="cuda").float() % 5 - 2) if pad else None
    v = framed((rows, rank), F32, pad, shift)
    lay = so.SFC_B_NK if nk else so.SFC_B_KN
    so.sfc_lora_down(x, a, ids, v, scales=scales, layout=lay)
    assert same(v, down(x, a, ids, scales, nk))
    need = so.sfc_lora_down_ws_size(rows, cols, rank, adapters)
    ws, again = framed((1, max(need // 4, 4)), F32), torch.empty_like(v)
    so.sfc_lora_down(x, a, ids, again, scales=scales, layout=lay, workspace=ws)
    assert torch.equal(again, v) and (need == 0) == bool(torch.isnan(ws).all())
    assert untouched_outside(v)


@pytest.mark.parametrize("rows,cols,rank,adapters", SHAPES)
@pytest.mark.parametrize("kind", ["rows", "runs", "one"])
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_up(so, rows, cols, rank, adapters, kind, nk, dtype, pad, shift):
    ids = make_ids(rows, adapters, rows + rank, kind)
    g = torch.Generator().manual_seed(3)
    v = framed((rows, rank), F32, pad, shift)
    v.copy_(torch.randint(-4000, 4001, (rows, rank), generator=g).float())
    b = small_ints((adapters, cols, rank) if nk else (adapters, rank, cols), 4, pad, shift, gap=3)
    base = framed((rows, cols), dtype, pad, shift)
    base.copy_(torch.randint(-200, 201, (rows, cols), generator=g).to(dtype))
    y = framed((rows, cols), dtype, pad + 1, shift)
    lay = so.SFC_B_NK if nk else so.SFC_B_KN
    so.sfc_lora_up(v, b, ids, y, base=base, layout=lay)
    want = up(v, b, ids, base, nk)
    assert same(y, want)
    assert untouched_outside(y)
    so.sfc_lora_up(v, b, ids, y, layout=lay)
    assert same(y, up(v, b, ids, torch.zeros_like(base), nk))
    so.sfc_lora_up(v, b, ids, base, base=base, layout=lay)
    assert same(base, want) and untouched_outside(base)


@pytest.mark.parametrize("rows,cols,rank,adapters", SHAPES)
@pytest.mark.parametrize("kind", ["rows", "runs", "one"])
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_weight_gradient(so, rows, cols, rank, adapters, kind, nk, dtype, pad, shift):
    ids = make_ids(rows, adapters, rows + rank, kind)
    z = small_ints((rows, cols), 5, pad, shift)
    g = torch.Generator().manual_seed(6)
    v = framed((rows, rank), F32, pad, shift)
    v.copy_(torch.randint(-500, 501, (rows, rank), generator=g).float())
    out = framed((adapters, cols, rank) if nk else (adapters, rank, cols), dtype, pad, shift, gap=2)
    lay = so.SFC_B_NK if nk else so.SFC_B_KN
    so.sfc_lora_wgrad(z, v, ids, out, layout=lay)
    need = so.sfc_lora_wgrad_ws_size(rows, cols, rank, adapters)
    ws = framed((1, max(need // 4, 4)), F32)
    again = torch.empty_like(out)
    so.sfc_lora_wgrad(z, v, ids, again, layout=lay, workspace=ws)
    assert torch.equal(again, out) and (need == 0) == bool(torch.isnan(ws).all())
    for a in range(adapters):
        t = torch.nonzero(ids == a)[:, 0]
        w = z[t].double().t() @ v[t].double()
        assert same(out[a], w if nk else w.t())
    assert untouched_outside(out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N,K,rank,adapters,kind", [(48, 300, 1030, 16, 12, "rows"), (700, 1000, 513, 40, 3, "runs"),
                                                         (1500, 520, 264, 200, 2, "one")])
def test_normal_values(so, rows, N, K, rank, adapters, kind, dtype):
    ids = make_ids(rows, adapters, 9, kind)
    x, dy = normals((rows, K), 1), normals((rows, N), 2, 1e-3)
    a, b = normals((adapters, rank, K), 3, K ** -0.5), normals((adapters, N, rank), 4, 0.02)
    scales = torch.rand(adapters, device="cuda") + 0.5
    base, dbase = normals((rows, N), 5, dtype=dtype), normals((rows, K), 6, 1e-3, dtype=dtype)
    v, u = torch.empty((rows, rank), device="cuda"), torch.empty((rows, rank), device="cuda")
    y, dx = torch.empty((rows, N), dtype=dtype, device="cuda"), torch.empty((rows, K), dtype=dtype, device="cuda")
    da, db = torch.empty_like(a, dtype=dtype), torch.empty_like(b, dtype=dtype)
    so.sfc_lora_down(x, a, ids, v, scales=scales)
    so.sfc_lora_up(v, b, ids, y, base=base)
    so.sfc_lora_down(dy, b, ids, u, scales=scales, layout=so.SFC_B_KN)
    so.sfc_lora_up(u, a, ids, dx, base=dbase, layout=so.SFC_B_KN)
    so.sfc_lora_wgrad(x, u, ids, da, layout=so.SFC_B_KN)
    so.sfc_lora_wgrad(dy, v, ids, db)
    assert close(v, down(x, a, ids, scales, True), down(x.abs(), a.abs(), ids, scales, True), K + 1, F32)
    assert close(u, down(dy, b, ids, scales, False), down(dy.abs(), b.abs(), ids, scales, False), N + 1, F32)
    # V to 16 bits: 2^-16 = 2^7 * 2^-23 of every product
    extra = 128 if dtype == BF16 else 0
    assert close(y, up(v, b, ids, base, True), up(v.abs(), b.abs(), ids, base.abs(), True), 3 * rank + 2 + extra, dtype)
    assert close(dx, up(u, a, ids, dbase, False), up(u.abs(), a.abs(), ids, dbase.abs(), False), 3 * rank + 2 + extra, dtype)
    for i in range(adapters):
        t = torch.nonzero(ids == i)[:, 0]
        for got, p, q in ((da[i], u[t].double(), x[t].double()), (db[i], dy[t].double(), v[t].double())):
            assert close(got, p.t() @ q, p.abs().t() @ q.abs(), 3 * len(t) + 2, dtype)


def test_empty_sides(so):
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    v = torch.full((4, 8), 3.0, device="cuda")
    so.sfc_lora_down(z(4, 0), z(2, 8, 0), ids, v)
    assert (v == 0).all()
    base = torch.randn((4, 9), device="cuda")
    y = torch.empty_like(base)
    so.sfc_lora_up(z(4, 0, dtype=F32), z(2, 9, 0), ids, y, base=base)
    assert torch.equal(y, base)
    g = torch.full((2, 9, 8), 5.0, device="cuda")
    so.sfc_lora_wgrad(z(0, 9), z(0, 8, dtype=F32), ids[:0], g)
    assert (g == 0).all()
    so.sfc_lora_down(z(0, 16), z(2, 8, 16), ids[:0], v[:0])
    so.sfc_lora_up(v[:0], z(2, 9, 8), ids[:0], y[:0])


def test_an_adapter_with_infinities_and_rows_with_nan(so):
    """Neither reaches another adapter's rows, nor a row of another request."""
    rows, K, N, rank, n = 40, 200, 150, 20, 4
    ids = torch.arange(rows, dtype=torch.int32, device="cuda") % (n + 1)
    x, a, b = small_ints((rows, K), 1), small_ints((n, rank, K), 2), small_ints((n, N, rank), 3)
    bad, row = 2, 6                                     # adapter, and a row of adapter 1
    clean = lambda t: torch.isfinite(t).all()           # noqa: E731
    for lay in (so.SFC_B_NK, so.SFC_B_KN):
        for value in (float("inf"), float("nan")):
            xx, aa, bb = x.clone(), a.clone(), b.clone()
            aa[bad], bb[bad], xx[row, 3] = value, value, value
            if lay == so.SFC_B_KN:
                aa, bb = aa.transpose(1, 2).contiguous(), bb.transpose(1, 2).contiguous()
            v = torch.empty((rows, rank), device="cuda")
            so.sfc_lora_down(xx, aa, ids, v, layout=lay)
            broken = (ids == bad) | (torch.arange(rows, device="cuda") == row)
            assert clean(v[~broken]) and not torch.isfinite(v[broken]).all(1).any()
            good = down(x, a, ids, None, True)
            assert same(v[~broken], good[~broken])
            for dtype in (F32, BF16):
                y = torch.empty((rows, N), dtype=dtype, device="cuda")
                so.sfc_lora_up(v, bb, ids, y, layout=lay)
                assert clean(y[~broken]) and not torch.isfinite(y[broken]).any()
            g = torch.empty((n, K, rank), device="cuda")
            so.sfc_lora_wgrad(xx, v, ids, g)
            assert clean(g[0]) and clean(g[3]) and not torch.isfinite(g[bad]).any() and not torch.isfinite(g[1, 3]).any()
