"""Experts' bf16 products and weight gradients on the GPU.

Operands are whole numbers whose products and sums fit 24 bits, so an fp32 result is exact and bf16 output
is its rounding, bit for bit; everything around the operands in memory is NaN.  Normal values: products are
exact, an fp32 sum of K of them in any order is within K * 2^-23 of the sum of magnitudes, bf16 output adds
2^-8 of the result."""
import numpy as np
import pytest
import torch

from rows_cases import BF16, DEPTHS, EXPERTS, F32, FEW, close, framed, normals, offsets_of, small_ints, untouched_outside

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def product(a, b, counts, layout_nk):
    """C in 64 bits: rows of a times the weights of their expert."""
    out, at = [], 0
    for e, n in enumerate(counts):
        w = b[e].double()
        out.append(a[at:at + n].double() @ (w.t() if layout_nk else w))
        at += n
    return torch.cat(out)


def same(got, want):
    """got holds want (exact in fp32) rounded to its type."""
    return torch.equal(got, want.float().to(got.dtype))


@pytest.mark.parametrize("counts,N,K", EXPERTS)
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_product(so, counts, N, K, nk, dtype, pad, shift):
    rows, E = sum(counts), len(counts)
    a = small_ints((rows, K), 1, pad, shift)
    b = small_ints((E, N, K) if nk else (E, K, N), 2, pad, shift, gap=5)
    c = framed((rows + 2, N), dtype, pad, shift)
    spare = framed((rows + 2, K), BF16)[:rows + 2]
    spare[:rows] = a
    so.sfc_moe_gemm_ex(spare if pad == 0 else a, b, offsets_of(counts), c if pad == 0 else c[:rows],
                       layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    torch.cuda.synchronize()
    assert same(c[:rows], product(a, b, counts, nk))
    if pad == 0:
        assert (c[rows:] == 0).all()                    # rows of no expert
    assert untouched_outside(c if pad == 0 else c[:rows])


@pytest.mark.parametrize("counts,N,K", [e for e in EXPERTS if sum(e[0]) > 0])
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("topk", [1, 3])
def test_product_of_rows_through_an_order(so, counts, N, K, nk, topk):
    rows, E, tokens = sum(counts), len(counts), 37
    rng = np.random.default_rng(rows + N)
    order = rng.integers(0, tokens * topk, rows).astype(np.int32)
    order[rng.random(rows) < 0.2] = rng.choice([-1, -(1 << 31), tokens * topk, (1 << 31) - 1])
    x = small_ints((tokens, K), 3, 5, 1)
    b = small_ints((E, N, K) if nk else (E, K, N), 4)
    c = framed((rows, N), F32, 2)
    so.sfc_moe_gemm_ex(x, b, offsets_of(counts), c, order=torch.from_numpy(order).cuda(), topk=topk,
                       layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    src = torch.from_numpy(np.where((order >= 0) & (order // topk < tokens), order // topk, tokens).astype(np.int64)).cuda()
    a = torch.cat([x, torch.zeros((1, K), dtype=BF16, device="cuda")])[src]
    assert same(c, product(a, b, counts, nk))
    assert untouched_outside(c)


@pytest.mark.parametrize("counts,N,K", FEW)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("topk", [0, 2])
def test_few_rows(so, counts, N, K, dtype, topk):
    """Operands of 16-byte pieces, a row behind the last segment, through an order (topk > 0) or not."""
    rows, E, tokens = sum(counts), len(counts), 19
    b = small_ints((E, N, K), 7, 8, 0, gap=16)
    c = framed((rows + 1, N), dtype, 3, 1)
    if topk:
        x = small_ints((tokens, K), 8, 16)
        rng = np.random.default_rng(rows + N)
        order = rng.integers(-1, tokens * topk + 2, rows + 1).astype(np.int32)
        src = torch.from_numpy(np.where((order >= 0) & (order // topk < tokens), order // topk, tokens).astype(np.int64)).cuda()
        a = torch.cat([x, torch.zeros((1, K), dtype=BF16, device="cuda")])[src]
        so.sfc_moe_gemm_ex(x, b, offsets_of(counts), c, order=torch.from_numpy(order).cuda(), topk=topk)
    else:
        a = small_ints((rows + 1, K), 8, 16)
        so.sfc_moe_gemm_ex(a, b, offsets_of(counts), c)
    if rows:
        assert same(c[:rows], product(a, b, counts, True))
    assert (c[rows:] == 0).all() and untouched_outside(c)


@pytest.mark.parametrize("counts,M,N", DEPTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_weight_gradient(so, counts, M, N, dtype, pad, shift):
    rows, E = sum(counts), len(counts)
    a, b = small_ints((rows, M), 5, pad, shift), small_ints((rows, N), 6, pad, shift)
    c = framed((E, M, N), dtype, pad, shift, gap=3)
    so.sfc_moe_wgrad_ex(a, b, offsets_of(counts), c)
    at = 0
    for e, n in enumerate(counts):
        assert same(c[e], a[at:at + n].double().t() @ b[at:at + n].double())
        at += n
    assert untouched_outside(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,N,K", [([100, 0, 300, 29], 520, 1030), ([2000, 1500, 900], 4096, 520)])
def test_normal_values(so, counts, N, K, dtype):
    rows, E = sum(counts), len(counts)
    x, w, dy = normals((rows, K), 7), normals((E, N, K), 8, 0.02), normals((rows, N), 9, 1e-3)
    offsets = offsets_of(counts)
    y, dx = torch.empty((rows, N), dtype=dtype, device="cuda"), torch.empty((rows, K), dtype=dtype, device="cuda")
    dw = torch.empty((E, N, K), dtype=dtype, device="cuda")
    so.sfc_moe_gemm_ex(x, w, offsets, y)
    so.sfc_moe_gemm_ex(dy, w, offsets, dx, layout=so.SFC_B_KN)
    so.sfc_moe_wgrad_ex(dy, x, offsets, dw)
    assert close(y, product(x, w, counts, True), product(x.abs(), w.abs(), counts, True), K, dtype)
    assert close(dx, product(dy, w, counts, False), product(dy.abs(), w.abs(), counts, False), N, dtype)
    at = 0
    for e, n in enumerate(counts):
        s, d = x[at:at + n].double(), dy[at:at + n].double()
        assert close(dw[e], d.t() @ s, d.abs().t() @ s.abs(), n, dtype)
        at += n


def test_offsets_outside_the_rows(so):
    """Bounds past the rows count as the nearest, rows before the first segment stay as they were."""
    a, b = small_ints((50, 40), 1), small_ints((3, 30, 40), 2)
    for bounds, segments in (([5, 20, 20, 40], [(5, 20), (20, 20), (20, 40)]), ([-7, 10, 60, 1 << 30], [(0, 10), (10, 50), (50, 50)])):
        offsets = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        c = torch.full((50, 30), 7.0, device="cuda")
        so.sfc_moe_gemm_ex(a, b, offsets, c)
        want = torch.zeros((50, 30), device="cuda")
        want[:segments[0][0]] = 7
        for e, (lo, hi) in enumerate(segments):
            want[lo:hi] = (a[lo:hi].double() @ b[e].double().t()).float()
        assert torch.equal(c, want)
        dw = torch.empty((3, 30, 40), device="cuda")
        dy = small_ints((50, 30), 3)
        so.sfc_moe_wgrad_ex(dy, a, offsets, dw)
        for e, (lo, hi) in enumerate(segments):
            assert torch.equal(dw[e], (dy[lo:hi].double().t() @ a[lo:hi].double()).float())


def test_infinities_stay_in_their_rows_and_experts(so):
    counts = [40, 0, 50, 30]
    a, b = small_ints((120, 200), 1), small_ints((4, 140, 200), 2)
    a[45, 3], a[46, 5] = float("inf"), float("nan")
    b[3, 7, 9] = float("inf")
    c = torch.empty((120, 140), device="cuda")
    so.sfc_moe_gemm_ex(a, b, offsets_of(counts), c)
    want = product(a, b, counts, True).float()
    assert torch.equal(torch.isnan(c), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(c), torch.nan_to_num(want))
    assert torch.isfinite(c[:45]).all() and torch.isfinite(c[47:90]).all()
    dw = torch.empty((4, 140, 200), device="cuda")
    dy = small_ints((120, 140), 4)
    so.sfc_moe_wgrad_ex(dy, a, offsets_of(counts), dw)
    assert torch.isfinite(dw[0]).all() and (dw[1] == 0).all() and torch.isfinite(dw[3]).all()
    assert not torch.isfinite(dw[2, :, 3]).any() and torch.isfinite(dw[2, :, :3]).all()
