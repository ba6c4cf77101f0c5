"""Infinities and NaN in the adapters' weights, rows and V, in batches that are taken in tiles: each reaches the sums that the
formula has it in and no others, and an infinite weight (or row of Z) times a finite V that is not 0 is an infinity, however few
bits V takes.  Whole numbers otherwise, so that finite sums are exact but
for tiny V among them: adding one to a whole number is a rounding, by up to 2^-23 of the sum so far (the matrix units do not
round to nearest), which is at most that of the magnitudes, as often as there are products: three of a V, and the base."""
import numpy as np
import pytest
import torch

from lora_cases import SPECIAL, TALL, agrees, product, special
from rows_cases import BF16, F32, framed, small_ints, untouched_outside

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
# finite values of one, two and three bf16 terms, of both signs, and some below the least normal number, below 2^-133 among them
FEW_BITS = [1.0, -1.0, 0.5, 257.0, -65537.0, 2.0 ** -100, -2.0 ** -130, 2.0 ** -133, 2.0 ** -140, -2.0 ** -149]


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def alternating(rows, n, seed):
    """Several adapters, and none, in every 16 rows; a run at the end."""
    ids = (np.arange(rows) * 7 // 3) % (n + 1)
    ids[-200:] = n - 1
    ids[np.random.default_rng(seed).random(rows) < 0.02] = -1
    return torch.from_numpy(ids.astype(np.int32)).cuda()


def low_nan():
    """A NaN whose payload lies in the lower half of its bits."""
    return torch.tensor([0x7F800001], dtype=torch.int32).view(torch.float32)[0]


def whole(rows, rank, most=200):
    g = torch.Generator().manual_seed(rows)
    return torch.randint(-most, most + 1, (rows, rank), generator=g).float().cuda()


@pytest.mark.parametrize("rows,cols,rank,n", SPECIAL)
@pytest.mark.parametrize("nk", [True, False])
def test_down(so, rows, cols, rank, n, nk):
    ids = alternating(rows, n, 1)
    x, a = small_ints((rows, cols), 1, 3, 1), small_ints((n, rank, cols), 2)
    special(x, 30, [INF, -INF, NAN], 3)
    if n > 1:
        special(a[n - 2], 4, [INF, NAN, -INF], 4)
    v = framed((rows, rank), F32, 1)
    so.sfc_lora_down(x, a if nk else a.transpose(1, 2).contiguous(), ids, v, layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    for i in range(n):
        t = torch.nonzero(ids == i)[:, 0]
        want, _ = product(x[t], a[i])
        assert agrees(v[t], want, 0.0)
    assert not v[(ids < 0) | (ids >= n)].any() and untouched_outside(v)


@pytest.mark.parametrize("rows,cols,rank,n", SPECIAL)
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("which", ["weights", "V", "both"])
def test_up(so, rows, cols, rank, n, nk, dtype, which):
    ids = alternating(rows, n, 1)
    v, b = whole(rows, rank), small_ints((n, cols, rank), 5)
    special(v, 200, FEW_BITS + [0.0], 6)
    if which != "weights":
        special(v, 12, [INF, -INF, NAN], 7)
        v[3, 0], v[rows - 2, rank - 1] = low_nan(), low_nan()
    if which != "V":
        special(b[0], 6, [INF, -INF, INF, NAN], 8)
        v[:, 0] = torch.tensor(FEW_BITS, device="cuda").repeat(rows // len(FEW_BITS) + 1)[:rows]
        b[0, cols // 2, 0], b[0, 0, 0] = INF, -INF
    base = small_ints((rows, cols), 9).to(dtype)
    y = framed((rows, cols), dtype, 1)
    so.sfc_lora_up(v, b if nk else b.transpose(1, 2).contiguous(), ids, y, base=base, layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    for i in range(n):
        t = torch.nonzero(ids == i)[:, 0]
        want, size = product(v[t], b[i])
        want += base[t].double()
        size += base[t].double().abs()
        # (below 2^-126, V has 2^-134 at the least)
        bound = (3 * rank + 1) * 2.0 ** -23 * size + 2.0 ** -134 * torch.where(torch.isfinite(b[i]), b[i].abs(), 0.0).sum(-1).double()
        # (bf16 results take V to 2^-16, and are rounded to 2^-8)
        bound = bound + 2.0 ** -16 * size + 2.0 ** -8 * (want.abs() + 2.0 ** -15 * size) if dtype == BF16 else bound
        assert agrees(y[t], want, bound)
    none = (ids < 0) | (ids >= n)
    assert torch.equal(y[none], base[none]) and untouched_outside(y)


@pytest.mark.parametrize("rows,cols,rank,n", TALL)
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_up_of_256_rows_to_a_workgroup(so, rows, cols, rank, n, nk, dtype):
    test_up(so, rows, cols, rank, n, nk, dtype, "both")


@pytest.mark.parametrize("rows,cols,rank,n", SPECIAL)
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("which", ["rows", "V", "both"])
def test_weight_gradient(so, rows, cols, rank, n, nk, which):
    ids = alternating(rows, n, 1)
    z, v = small_ints((rows, cols), 1, 3, 1), whole(rows, rank, 20)
    if which != "V":
        special(z, 3, [INF, -INF, NAN], 3)
        special(z[-150:], 2, [INF, -INF], 4)           # (rows of the last adapter)
    if which != "rows":
        special(v, 4, [INF, NAN, -INF, low_nan()], 5)
    tiny = torch.isinf(z).any(1) & (torch.arange(rows, device="cuda") % 2 == 0)
    v[tiny, 0] = 2.0 ** -140
    g = framed((n, cols, rank) if nk else (n, rank, cols), F32, 1)
    so.sfc_lora_wgrad(z, v, ids, g, layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    for i in range(n):
        t = torch.nonzero(ids == i)[:, 0]
        want, size = product(z[t].t(), v[t].t())
        bound = 3 * len(t) * 2.0 ** -23 * size + 2.0 ** -134 * torch.where(torch.isfinite(z[t]), z[t].abs(), 0.0).sum(0).double()[:, None]
        assert agrees(g[i] if nk else g[i].t(), want, bound)
    assert untouched_outside(g)


@pytest.mark.parametrize("rows,cols,rank,n", [(70_001, 40, 9, 2), (140_000, 300, 20, 1), (66_000, 6, 5, 3), (131_100, 70, 8, 1030)])
@pytest.mark.parametrize("nk", [True, False])
def test_weight_gradient_of_more_rows_than_are_listed_at_a_time(so, rows, cols, rank, n, nk):
    """Infinite Z in the first rows and the last, times V of which later terms are 0."""
    ids = (torch.arange(rows, device="cuda") // 50 % n).to(torch.int32)
    z, v = small_ints((rows, cols), 1, most=1), torch.ones((rows, rank), device="cuda")
    v[::2] = -2.0
    z[70, cols // 2], z[rows - 3, 1] = INF, -INF
    g = torch.full((n, cols, rank) if nk else (n, rank, cols), 5.0, device="cuda")
    so.sfc_lora_wgrad(z, v, ids, g, layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    for i in {0, n - 1, int(ids[70]), int(ids[rows - 3])}:
        t = torch.nonzero(ids == i)[:, 0]
        want, _ = product(z[t].t(), v[t].t())
        assert agrees(g[i] if nk else g[i].t(), want, 0.0)
    assert torch.isinf(g).sum() == 2 * rank and not torch.isnan(g).any()


@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_gives_the_same_alone_and_in_a_batch(so, nk, dtype):
    """Infinities of an adapter whose V are powers of two: as one row and among 4200."""
    rows, cols, rank, n = 4200, 80, 16, 2
    ids = torch.arange(rows, dtype=torch.int32, device="cuda") % n
    v, b = torch.exp2(whole(rows, rank, 20)), small_ints((n, cols, rank), 5)
    b[1, ::3, 4], b[1, 1::3, 7] = INF, -INF
    w, lay = b if nk else b.transpose(1, 2).contiguous(), so.SFC_B_NK if nk else so.SFC_B_KN
    y, alone = torch.empty((rows, cols), dtype=dtype, device="cuda"), torch.empty((7, cols), dtype=dtype, device="cuda")
    so.sfc_lora_up(v, w, ids, y, layout=lay)
    so.sfc_lora_up(v[:7], w, ids[:7], alone, layout=lay)
    assert torch.isinf(alone[1::2, ::3]).all() and not torch.isnan(alone).any()
    infinite = torch.isinf(alone)
    assert torch.equal(y[:7][infinite], alone[infinite]) and torch.isfinite(y[:7][~infinite]).all()
    assert not torch.isnan(y).any()
