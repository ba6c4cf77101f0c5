"""Matrices longer than one launch takes (2^23 rows or tokens, 2^26 rows to clear, 2^22 blocks of
columns): every row, token and column of them, and past 2^32 threads in all."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, I32, U8 = torch.float32, torch.bfloat16, torch.int32, torch.uint8
ROWS = (1 << 24) + 33                # three launches


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def spread(n, below, seed):
    """n whole numbers 0 .. below - 1, all over."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, below, (n,), generator=g, device="cuda", dtype=I32)


def test_dispatch(so):
    x = torch.randn((1000, 5), device="cuda").to(BF16)
    order = spread(ROWS, 3003, 1) - 2
    xs = torch.full((ROWS, 5), 9.0, dtype=BF16, device="cuda")
    so.sfc_moe_dispatch(x, order, xs, topk=3)
    want = x[(order.long() // 3).clamp(0, 999)] * ((order >= 0) & (order < 3000))[:, None]
    assert torch.equal(xs, want)


def test_combine(so):
    ys = torch.randn((1000, 3), device="cuda")
    pos = spread(ROWS * 2, 1001, 2) - 1
    w = torch.rand((ROWS, 2), device="cuda")
    y = torch.empty((ROWS, 3), device="cuda")
    so.sfc_moe_combine(ys, pos, y, weights=w)
    p = pos.view(ROWS, 2).long()
    terms = ys.double()[p.clamp(min=0)] * (w.double() * (p >= 0))[..., None]
    assert ((y - terms.sum(1)).abs() <= 3 * 2.0 ** -23 * terms.abs().sum(1)).all()


# (the second: 2^32 threads and more in all)
@pytest.mark.parametrize("tokens,spare,cols", [((1 << 23) + 5, 1 << 26, 2), ((1 << 28) + 3, 70, 1)])
def test_gradient_of_combine(so, tokens, spare, cols):
    rows = tokens + spare
    order = torch.full((rows,), -1, dtype=I32, device="cuda")
    pos = torch.arange(rows - 1, rows - 1 - tokens, -1, dtype=I32, device="cuda")     # the last rows, backwards
    order[rows - tokens:] = torch.arange(tokens - 1, -1, -1, dtype=I32, device="cuda")
    dy, ys = torch.randn((tokens, cols), device="cuda"), torch.randn((rows, cols), device="cuda")
    w = torch.rand((tokens,), device="cuda")
    dys, dw = torch.full((rows, cols), 9.0, device="cuda"), torch.full((tokens,), 9.0, device="cuda")
    so.sfc_moe_combine_grad(dy, ys, order, pos, w, dys, dw)
    assert (dys[:rows - tokens] == 0).all()
    assert torch.equal(dys[rows - tokens:].flip(0), dy * w[:, None])
    terms = dy.double() * ys[rows - tokens:].flip(0)
    assert ((dw - terms.sum(1)).abs() <= (cols + 1) * 2.0 ** -23 * terms.abs().sum(1)).all()


@pytest.mark.parametrize("cols", [5, 33])
def test_quant_along_rows_and_back(so, cols):
    """Row by row the same as a short matrix that holds the same rows."""
    x = torch.randn((1000, cols), device="cuda").to(BF16)
    q0, s0 = so.mx4_empty(1000, cols)
    so.sfc_mx4_quant(x, q0, s0)
    pick = spread(ROWS, 1000, 3)
    q, s = so.mx4_empty(ROWS, cols)
    so.sfc_mx4_quant(x[pick.long()], q, s)
    assert torch.equal(q, q0[pick.long()]) and torch.equal(s, s0[pick.long()])
    q.fill_(7)
    so.sfc_mx4_quant(x, q, s, order=pick * 2 + 1, topk=2)
    assert torch.equal(q, q0[pick.long()]) and torch.equal(s, s0[pick.long()])
    y0, y = torch.empty((1000, cols), device="cuda"), torch.empty((ROWS, cols), device="cuda")
    so.sfc_mx4_dequant(q0, s0, y0)
    so.sfc_mx4_dequant(q, s, y)
    assert torch.equal(y, y0[pick.long()])


# one block of rows: 2^29 columns a launch; 3 blocks with an order
@pytest.mark.parametrize("rows,cols,topk", [(1, (1 << 29) + 300, 0), (300, ((1 << 22) // 3 + 5) * 128 + 77, 2)])
def test_quant_along_columns(so, rows, cols, topk):
    x = torch.randn((1 if topk else rows, cols), device="cuda", dtype=BF16)
    order = torch.arange(rows, device="cuda", dtype=I32) % 3 if topk else None      # slots 0 and 1: row 0; slot 2: none
    qt, st = so.mx4_empty(cols, rows)
    so.sfc_mx4_quant(x, None, None, qt, st, order=order, topk=topk or 1)
    edge = (1 << 22) // -(-rows // 128) * 128
    for lo, hi in ((0, 500), (edge - 300, min(edge + 300, cols)), (cols - 200, cols)):
        part = so.mx4_empty(hi - lo, rows)
        so.sfc_mx4_quant(x[:, lo:hi].clone(), None, None, *part, order=order, topk=topk or 1)
        assert torch.equal(qt[lo:hi], part[0]) and torch.equal(st[lo:hi], part[1])


def test_product_of_many_columns(so):
    """Past 2^28 columns few rows run on the block kernel."""
    M, N, K = 17, (1 << 28) + 100, 32
    g = torch.Generator(device="cuda").manual_seed(4)
    few = torch.randint(0, 256, (1024, 16), generator=g, device="cuda", dtype=U8)
    B = torch.zeros((N, 16), device="cuda", dtype=U8)
    B[:1024] = few
    B[-1024:] = few
    Bs = torch.full((N, 4), 255, device="cuda", dtype=U8)[:, :1]
    Bs.fill_(127)
    A, As = torch.randint(0, 256, (M, 16), generator=g, device="cuda", dtype=U8), torch.full((M, 4), 127, device="cuda", dtype=U8)[:, :1]
    C = torch.empty((M, N), device="cuda", dtype=BF16)
    so.sfc_gemm_mx4_ex(A, As, B, Bs, C)
    want = torch.empty((M, 1024), device="cuda", dtype=BF16)
    so.sfc_gemm_mx4_ex(A, As, few, torch.full((1024, 4), 127, device="cuda", dtype=U8)[:, :1], want)     # sums are exact
    assert torch.equal(C[:, :1024], want) and torch.equal(C[:, -1024:], want)
    assert (C[:, 1024:-1024] == 0).all()
