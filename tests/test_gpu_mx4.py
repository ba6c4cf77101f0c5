"""4-bit operators on the GPU: quantisation bit by bit against the oracle, products against 64
bits, at the sizes, strides, scales and special values where they can go wrong.

Bar of a product: every a * b and every scale is exact, so an fp32 sum of K terms, in any
order, is within K * 2^-23 * sum |a b| of the exact one (2^-23: adders that truncate); bf16
output adds 2^-8 of the result.  Where all partial sums fit 24 bits the result is exact."""
import numpy as np
import pytest
import torch

from mx4_cases import PRODUCTS
from oracle import mx4

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def host(x):
    return x.float().cpu().numpy().astype(np.float64)


def padded_mx4(rows, cols, pad=0):
    """A pair whose rows lie `pad` values (a multiple of 128) further apart than they need."""
    b = -(-cols // 32)
    q = torch.zeros((rows, 16 * b + pad // 2), dtype=torch.uint8, device="cuda")
    s = torch.zeros((rows, (b + 3) // 4 * 4 + pad // 32), dtype=torch.uint8, device="cuda")
    return q, s, q[:, :16 * b], s[:, :b]


def inputs(rows, cols, dtype, seed, ld=None, offset=0):
    g = torch.Generator().manual_seed(seed)
    ld = cols if ld is None else ld
    flat = torch.randn((rows * ld + offset,), generator=g) * torch.exp2(4 * torch.randn((rows * ld + offset,), generator=g))
    flat[torch.rand(flat.shape, generator=g) < 0.05] = 0
    flat = flat.to(dtype).cuda()
    return flat[offset:].view(rows, ld)[:, :cols]


SHAPES = [(1, 1), (1, 32), (3, 31), (5, 33), (16, 4096), (33, 70), (257, 129), (300, 1000), (64, 8200), (1025, 96)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("ld,offset", [(0, 0), (7, 1)])
def test_quant_bits(so, dtype, rows, cols, ld, offset):
    x = inputs(rows, cols, dtype, rows * 1000 + cols, cols + ld, offset)
    q, s = so.mx4_empty(rows, cols)
    qt, st = so.mx4_empty(cols, rows)
    for t in (q, s, qt, st):
        t.fill_(0xAA)
    so.sfc_mx4_quant(x, q, s, qt, st)
    torch.cuda.synchronize()
    c, e = mx4.quantise(host(x))
    assert (s.cpu().numpy() == e).all()
    assert (q.cpu().numpy() == mx4.pack(c)).all()
    c, e = mx4.quantise(host(x).T)
    assert (st.cpu().numpy() == e).all()
    assert (qt.cpu().numpy() == mx4.pack(c)).all()
    # one output at a time gives the same
    q2, s2 = so.mx4_empty(rows, cols)
    qt2, st2 = so.mx4_empty(cols, rows)
    so.sfc_mx4_quant(x, q2, s2)
    so.sfc_mx4_quant(x, None, None, qt2, st2)
    assert torch.equal(q, q2) and torch.equal(s, s2) and torch.equal(qt, qt2) and torch.equal(st, st2)


def test_quant_every_bf16_value(so):
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF16).cuda()
    # blocks of 32: a fixed largest magnitude (sets the scale) and 31 others below it or above
    for top in (1.0, 2.0 ** -120, 2.0 ** -126, 2.0 ** -130, 2.0 ** 100, 3.0e38):
        x = torch.full((2115, 32), 0.0, dtype=BF16, device="cuda")
        flat = torch.zeros(2115 * 31, dtype=BF16, device="cuda")
        flat[:65536] = bits
        flat = torch.where(flat.float().abs() <= top, flat, torch.zeros_like(flat))
        x[:, 1:] = flat.view(2115, 31)
        x[:, 0] = top
        q, s = so.mx4_empty(2115, 32)
        so.sfc_mx4_quant(x, q, s)
        c, e = mx4.quantise(host(x))
        assert (s.cpu().numpy() == e).all() and (q.cpu().numpy() == mx4.pack(c)).all(), top


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_special_values(so, dtype):
    x = inputs(40, 200, dtype, 5).clone()
    x[3, 40] = float("inf")
    x[4, 70] = float("-inf")
    x[5, 199] = float("nan")
    x[6] = 0
    x[7] = -0.0
    x[8] = torch.finfo(dtype).min
    x[9] = torch.finfo(dtype).tiny
    x[10] = torch.finfo(dtype).smallest_normal / 4
    q, s = so.mx4_empty(40, 200)
    qt, st = so.mx4_empty(200, 40)
    so.sfc_mx4_quant(x, q, s, qt, st)
    for (a, b, ref, n) in ((q, s, host(x), 200), (qt, st, host(x).T, 40)):
        c, e = mx4.quantise(ref)
        assert (b.cpu().numpy() == e).all()
        for dt in (F32, BF16):
            y = torch.empty((a.shape[0], n), dtype=dt, device="cuda")
            so.sfc_mx4_dequant(a, b, y)
            assert np.array_equal(host(y), mx4.values(c, e)[:, :n], equal_nan=True)


@pytest.mark.parametrize("rows,cols,topk,rows_out", [(7, 100, 2, 40), (300, 257, 4, 999), (1, 32, 1, 5)])
def test_quant_through_an_order(so, rows, cols, topk, rows_out):
    x = inputs(rows, cols, BF16, 9)
    g = torch.Generator().manual_seed(1)
    order = torch.randint(-2, rows * topk + 3, (rows_out,), generator=g, dtype=torch.int32)
    ref = np.zeros((rows_out, cols))
    for p, o in enumerate(order.tolist()):
        if 0 <= o < rows * topk:
            ref[p] = host(x)[o // topk]
    q, s = so.mx4_empty(rows_out, cols)
    qt, st = so.mx4_empty(cols, rows_out)
    so.sfc_mx4_quant(x, q, s, qt, st, order=order.cuda(), topk=topk)
    for (a, b, r) in ((q, s, ref), (qt, st, ref.T)):
        c, e = mx4.quantise(r)
        assert (b.cpu().numpy() == e).all() and (a.cpu().numpy() == mx4.pack(c)).all()


# (256 rows to a workgroup once those fill half of the CUs)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,ld,offset", [(2100, 2570, 7, 1), (4097, 1300, 0, 0), (33000, 130, 0, 0), (200, 17000, 3, 0)])
def test_quant_bits_of_large_matrices(so, dtype, rows, cols, ld, offset):
    test_quant_bits(so, dtype, rows, cols, ld, offset)


def test_quant_of_many_rows_through_an_order(so):
    test_quant_through_an_order(so, 40, 4100, 30, 1100)


def test_quant_writes_its_own_bytes_only(so):
    x = inputs(70, 100, BF16, 2)
    q, s, qv, sv = padded_mx4(70, 100, 128)
    qt, st, qtv, stv = padded_mx4(100, 70, 128)
    for t in (q, s, qt, st):
        t.fill_(0x5A)
    so.sfc_mx4_quant(x, qv, sv, qtv, stv)
    assert (q[:, 64:] == 0x5A).all() and (s[:, 4:] == 0x5A).all()
    assert (qt[:, 48:] == 0x5A).all() and (st[:, 3:] == 0x5A).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 7, 8, 31, 100, 4096])
def test_dequant_writes_inside_only(so, dtype, cols):
    rng = np.random.default_rng(cols)
    b = -(-cols // 32)
    c = rng.integers(0, 16, (9, 32 * b), dtype=np.uint8)
    e = rng.integers(0, 255, (9, b), dtype=np.uint8)
    if dtype == F32:
        e = np.minimum(e, 251)
    q, s = so.mx4_empty(9, cols)
    q.copy_(torch.from_numpy(mx4.pack(c)))
    s.copy_(torch.from_numpy(e))
    full = torch.full((9, cols + 5), 77.0, dtype=dtype, device="cuda")
    so.sfc_mx4_dequant(q, s, full[:, 1:1 + cols])
    want = mx4.values(c, e)[:, :cols]
    got = host(full)
    assert (got[:, 0] == 77).all() and (got[:, 1 + cols:] == 77).all()
    big = np.abs(want) > 3.39e38
    assert np.array_equal(got[:, 1:1 + cols][~big], want[~big]) and np.isinf(got[:, 1:1 + cols][big]).all()


# ---- products ---------------------------------------------------------------------------------


def operand(rows, K, seed, lo=127, hi=128, pad=0):
    """Random codes and scale codes lo .. hi: (codes, scales, float64 values on the GPU)."""
    rng = np.random.default_rng(seed)
    c = rng.integers(0, 16, (rows, K), dtype=np.uint8)
    e = rng.integers(lo, hi + 1, (rows, K // 32), dtype=np.uint8)
    full_q, full_s, q, s = padded_mx4(rows, K, pad)
    full_q.fill_(0x77)
    full_s.fill_(0xFF)                   # padding bytes hold NaN scales: none may be used
    q.copy_(torch.from_numpy(mx4.pack(c)))
    s.copy_(torch.from_numpy(e))
    return q, s, torch.from_numpy(mx4.values(c, e)).cuda()


def check(C, a, b, K, exact):
    want = a @ b.t()
    got = C.double()
    if exact:
        if C.dtype == BF16:
            want = want.float().to(BF16).double()
        assert torch.equal(got, want)
        return
    bound = K * 2.0 ** -23 * (a.abs() @ b.abs().t())
    if C.dtype == BF16:
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [shape for shape, _ in PRODUCTS])
def test_product_exact(so, M, N, K, out):
    # |a b| <= 36 * 4 in steps of 1/4: sums of up to 2^24 / (4 * 144) = 29127 terms are exact
    assert K <= 29127
    A, As, a = operand(M, K, M + 7 * K)
    B, Bs, b = operand(N, K, N + 3 * K)
    C = torch.full((M, N + 3), 99.0, dtype=out, device="cuda")
    so.sfc_gemm_mx4_ex(A, As, B, Bs, C[:, 1:1 + N])
    assert (C[:, 0] == 99).all() and (C[:, 1 + N:] == 99).all()
    check(C[:, 1:1 + N], a, b, K, True)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(5, 300, 4096), (16, 4200, 12000 // 32 * 32), (64, 64, 1056), (200, 300, 4096), (128, 256, 8192), (4000, 4090, 3136)])
def test_product_wide_scales(so, M, N, K, out):
    A, As, a = operand(M, K, 11, 100, 150, 128)
    B, Bs, b = operand(N, K, 12, 100, 150, 256)
    C = torch.empty((M, N), dtype=out, device="cuda")
    so.sfc_gemm_mx4_ex(A, As, B, Bs, C)
    check(C, a, b, K, False)
    again = torch.empty_like(C)
    so.sfc_gemm_mx4_ex(A, As, B, Bs, again)
    assert torch.equal(C, again)


@pytest.mark.parametrize("M,N,K", [(4, 70, 1056), (9, 4200, 9056), (20, 70, 1056), (150, 140, 1056), (4000, 4090, 3136)])
def test_nan_scales_reach_their_row_and_column_only(so, M, N, K):
    A, As, a = operand(M, K, 1)
    B, Bs, b = operand(N, K, 2)
    As[M // 2, K // 32 - 1] = 255
    Bs[N - 1, 0] = 255
    A[M // 2] = 0                        # zeros under a NaN scale are NaN
    C = torch.empty((M, N), dtype=F32, device="cuda")
    so.sfc_gemm_mx4_ex(A, As, B, Bs, C)
    nan = torch.isnan(C)
    want = torch.zeros_like(nan)
    want[M // 2] = True
    want[:, N - 1] = True
    assert torch.equal(nan, want)
    a[M // 2] = 0
    keep = ~want
    assert torch.equal(C.double()[keep], (a @ b.t())[keep])


@pytest.mark.parametrize("M,N", [(1, 5), (70, 200)])
def test_empty_sums_are_zero(so, M, N):
    A, As = so.mx4_empty(M, 0)
    B, Bs = so.mx4_empty(N, 0)
    for out in (F32, BF16):
        C = torch.full((M, N), 5.0, dtype=out, device="cuda")
        so.sfc_gemm_mx4_ex(A, As, B, Bs, C)
        assert (C == 0).all()
        C.fill_(5)
        so.sfc_mx4_linear(torch.empty((M, 0), dtype=BF16, device="cuda"), B, Bs, C)
        assert (C == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(1, 256, 4096), (16, 100, 77), (9, 300, 2050), (16, 9000, 4000), (3, 200, 4100),
                                   (50, 333, 2047), (333, 500, 100), (128, 128, 8000), (2100, 4100, 520)])
def test_linear_is_quantisation_and_product(so, M, N, K, dtype):
    x = inputs(M, K, dtype, 3, K + 5, 1)
    Kp = -(-K // 32) * 32
    W, Ws, w = operand(N, Kp, 4)
    for out in (F32, BF16):
        y = torch.empty((M, N), dtype=out, device="cuda")
        so.sfc_mx4_linear(x, W, Ws, y)
        q, s = so.mx4_empty(M, K)
        so.sfc_mx4_quant(x, q, s)
        z = torch.empty_like(y)
        so.sfc_gemm_mx4_ex(q, s, W, Ws, z)
        assert torch.equal(y, z)
        xv = torch.from_numpy(mx4.values(*mx4.quantise(host(x)))).cuda()
        check(y, xv, w, Kp, False)


def test_gradients_are_products_of_the_transposed_operands(so):
    """dx = dy W and dW = dy^T x against the formulas on the quantised values, and dW against
    differences of the loss sum(dy * (x W^T)) in W, which is linear in W."""
    M, N, K = 96, 160, 224
    x, dy, w = (inputs(r, c, BF16, i) for i, (r, c) in enumerate(((M, K), (M, N), (N, K))))
    dq, dt, wt, xt = so.mx4_empty(M, N), so.mx4_empty(N, M), so.mx4_empty(K, N), so.mx4_empty(K, M)
    so.sfc_mx4_quant(dy, *dq, *dt)
    so.sfc_mx4_quant(w, None, None, *wt)
    so.sfc_mx4_quant(x, None, None, *xt)
    dx, dw = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda")
    so.sfc_gemm_mx4_ex(*dq, *wt, dx)
    so.sfc_gemm_mx4_ex(*dt, *xt, dw)
    v = lambda t: torch.from_numpy(mx4.values(*mx4.quantise(host(t)))).cuda()
    vt = lambda t: torch.from_numpy(mx4.values(*mx4.quantise(host(t).T))).cuda()
    check(dx, v(dy), vt(w), N, False)
    check(dw, vt(dy), vt(x), M, False)
    x64, dy64 = vt(x).t(), vt(dy).t()
    w64 = w.double()
    loss = lambda m: (dy64 * (x64 @ m.t())).sum()
    for n, k in ((0, 0), (17, 100), (159, 223)):
        step = torch.zeros_like(w64)
        step[n, k] = 1.0
        diff = (loss(w64 + step) - loss(w64 - step)) / 2
        scale = (dy64.abs().t() @ x64.abs())[n, k] + 1e-9 * loss(w64.abs()).abs()
        assert abs(dw[n, k].double() - diff) <= (M * 2.0 ** -23) * scale + 1e-9 * (dy64.abs() * (x64.abs() @ w64.abs().t())).sum()


def test_a_long_row_passes_32_bit_offsets(so):
    # codes of A alone are 4.3 GB: rows past byte offset 2^32
    M, K, N = 70000, 131072, 48
    q = torch.zeros((M, K // 2), dtype=torch.uint8, device="cuda")
    s = torch.full((M, K // 32), 127, dtype=torch.uint8, device="cuda")
    rows = torch.tensor([0, 1, 32767, 32768, 65535, 65536, 65537, M - 1], device="cuda")
    q[rows] = torch.randint(0, 256, (rows.numel(), K // 2), dtype=torch.uint8, device="cuda")
    B, Bs, b = operand(N, K, 8, 127, 127)
    C = torch.empty((M, N), dtype=F32, device="cuda")
    so.sfc_gemm_mx4_ex(q, s, B, Bs, C)
    a = torch.from_numpy(mx4.GRID[mx4.unpack(q[rows].cpu().numpy())]).cuda()
    # steps of 1/4, |a b| <= 36: the running sums stay far below 2^24 / 4
    assert torch.equal(C[rows].double(), a @ b.t())
    other = torch.ones(M, dtype=torch.bool, device="cuda")
    other[rows] = False
    assert (C[other] == 0).all()


def test_streams_and_graphs(so):
    """Calls on two streams (workspaces of their own), and a recorded call replayed between eager ones."""
    M, N, K = 120, 130, 8192                   # layers: copies in library memory
    x = [inputs(M, K, BF16, i) for i in range(2)]
    W, Ws, w = operand(N, K, 4)
    want = []
    for i in range(2):
        y = torch.empty((M, N), device="cuda")
        so.sfc_mx4_linear(x[i], W, Ws, y)
        want.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.empty((M, N), device="cuda") for _ in range(2)]
    for _ in range(5):
        for i in range(2):
            so.sfc_mx4_linear(x[i], W, Ws, got[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    static = x[0].clone()
    out = torch.empty((M, N), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        so.sfc_mx4_linear(static, W, Ws, out)
    for i in (1, 0, 1):
        static.copy_(x[i])
        out.fill_(3)
        graph.replay()
        y = torch.empty((M, N), device="cuda")
        so.sfc_mx4_linear(x[1 - i], W, Ws, y)
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]) and torch.equal(y, want[1 - i])
