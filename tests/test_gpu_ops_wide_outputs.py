"""Row operators whose outputs are 32 MB and more: their stores go past the caches, by kernel variants of
their own.  Odd columns and leading dimensions, dropped slots and padding rows, all values checked.

Bars as in test_gpu_moe: a sum of k rows within (k + 1) * 2^-23 of the sum of magnitudes, a dot product
over D terms within (D + 1) * 2^-23, products rounded once; bf16 adds 2^-8 of the result."""
import pytest
import torch

from oracle import mx4
from test_gpu_moe import routing, sort

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
MB = 1 << 20


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def rows_of(n, cols, dtype, seed, pad=1):
    """n x cols values in rows `pad` elements further apart, from one element into the allocation."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((n, cols + pad), generator=g, device="cuda").to(dtype)[:, pad:]


def framed(n, cols, dtype):
    full = torch.full((n, cols + 2), 9.0, dtype=dtype, device="cuda")
    return full, full[:, 1:1 + cols]


def whole(full, cols):
    return bool((full[:, 0] == 9).all() and (full[:, 1 + cols:] == 9).all())


def size(t):
    return t.shape[0] * t.shape[1] * t.element_size()


def tokens(D, dtype, topk, mb):
    """As many as give an output of a little more than `mb` MB."""
    return mb * MB // (D * topk * (2 if dtype == BF16 else 4)) + 5


# 16, 64 and 256 lanes to a token; fp32 outputs of 128 MB and more stay in the caches
@pytest.mark.parametrize("dtype,mb", [(F32, 33), (F32, 129), (BF16, 33), (BF16, 129)])
@pytest.mark.parametrize("D", [63, 256, 257, 2047, 2049, 4103])
def test_gradient_of_combine(so, dtype, mb, D):
    k, E = 2, 8
    T = tokens(D, dtype, k, mb)
    ids = routing_of(T, k, E, D, 0.05)
    offsets, order, pos = sort(so, ids, E, 32)
    rows = order.numel()
    dy, ys = rows_of(T, D, dtype, 1), rows_of(rows, D, dtype, 2)
    w = torch.rand((T, k), device="cuda")
    full, dys = framed(rows, D, dtype)
    assert size(dys) >= 32 * MB and (size(dys) >= 128 * MB) == (mb == 129)
    dw = torch.full((T, k), 9.0, device="cuda")
    so.sfc_moe_combine_grad(dy, ys, order, pos, w, dys, dw)
    o, p = order.long(), pos.view(T, k).long()
    ref = dy.double()[o.clamp(min=0) // k] * torch.where(o >= 0, w.double().view(-1)[o.clamp(min=0)], 0.0)[:, None]
    assert ((dys.double() - ref).abs() <= (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * ref.abs()).all() and whole(full, D)
    del ref
    for j in range(k):
        terms = dy.double() * ys.double()[p[:, j].clamp(min=0)] * (p[:, j] >= 0)[:, None]
        assert ((dw[:, j].double() - terms.sum(1)).abs() <= (D + 1) * 2.0 ** -23 * terms.abs().sum(1)).all()


def routing_of(T, k, E, seed, dropped):
    """routing() of test_gpu_moe draws token by token; for many tokens a block of its rows repeats."""
    import numpy as np
    return np.resize(routing(min(T, 4001), k, E, seed, 0.5, dropped), (T, k))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [63, 1025, 4103])
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(so, dtype, D, weighted):
    k, E = 3, 8
    T = tokens(D, dtype, 1, 33)
    offsets, order, pos = sort(so, routing_of(T, k, E, D, 0.1), E, 16)
    ys = rows_of(order.numel(), D, dtype, 3)
    w = torch.rand((T, k), device="cuda") if weighted else None
    full, y = framed(T, D, dtype)
    assert size(y) >= 32 * MB
    so.sfc_moe_combine(ys, pos, y, weights=w)
    p = pos.view(T, k).long()
    ref, mag = (torch.zeros((T, D), dtype=torch.float64, device="cuda") for _ in range(2))
    for j in range(k):
        terms = ys.double()[p[:, j].clamp(min=0)] * (p[:, j] >= 0)[:, None] * (w[:, j].double()[:, None] if weighted else 1.0)
        ref += terms
        mag += terms.abs()
    bound = (k + 1) * 2.0 ** -23 * mag
    if dtype == BF16:
        bound = bound + 2.0 ** -8 * (ref.abs() + bound)
    assert ((y.double() - ref).abs() <= bound).all() and whole(full, D)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [63, 1025, 4103])
@pytest.mark.parametrize("weighted", [True, False])
def test_dispatch(so, dtype, D, weighted):
    k, E = 2, 8
    T = tokens(D, dtype, k, 33)
    offsets, order, pos = sort(so, routing_of(T, k, E, D, 0.1), E, 16)
    x, w = rows_of(T, D, dtype, 4), torch.rand((T, k), device="cuda")
    full, xs = framed(order.numel(), D, dtype)
    assert size(xs) >= 32 * MB
    so.sfc_moe_dispatch(x, order, xs, topk=k, weights=w if weighted else None)
    o = order.long()
    ref = x.double()[o.clamp(min=0) // k] * (o >= 0)[:, None]
    if weighted:
        ref = ref * w.double().view(-1)[o.clamp(min=0)][:, None]
        assert ((xs.double() - ref).abs() <= (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * ref.abs()).all()
    else:
        assert torch.equal(xs.double(), ref)
    assert whole(full, D)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [63, 1025, 4103])
def test_dequant(so, dtype, cols):
    rows = tokens(cols, dtype, 1, 33)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, s = so.mx4_empty(rows, cols)
    q.copy_(torch.randint(0, 256, q.shape, generator=g, device="cuda", dtype=torch.uint8))
    s.copy_(torch.randint(100, 150, s.shape, generator=g, device="cuda", dtype=torch.uint8))
    s[::97, 0] = 255
    full, y = framed(rows, cols, dtype)
    assert size(y) >= 32 * MB
    so.sfc_mx4_dequant(q, s, y)
    code = torch.stack((q & 15, q >> 4), dim=-1).reshape(rows, -1).long()
    value = torch.from_numpy(mx4.GRID).cuda()[code] * torch.from_numpy(mx4.e8m0_value(range(256))).cuda()[s.long()].repeat_interleave(32, 1)
    # E2M1 times a power of two is a bf16 value
    assert torch.equal(torch.nan_to_num(y.double(), nan=7e77), torch.nan_to_num(value[:, :cols], nan=7e77)) and whole(full, cols)
