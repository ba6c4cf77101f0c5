"""The row operators of the experts where tokens, rows or columns run out: no tokens at all, rows that
are no multiple of what a workgroup takes; nothing outside the arrays is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def framed(rows, cols, dtype):
    """(rows x cols inside, all of it): 20 rows before and behind, a column on each side."""
    full = torch.full((rows + 40, cols + 2), 9.0, dtype=dtype, device="cuda")
    return full[20:20 + rows, 1:1 + cols], full


def frame_is_whole(full, rows, cols):
    inside = torch.zeros_like(full, dtype=torch.bool)
    inside[20:20 + rows, 1:1 + cols] = True
    return bool((full[~inside] == 9).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 4, 15, 16, 17, 31, 61])
@pytest.mark.parametrize("cols", [1, 64, 300, 2050])
def test_no_tokens(so, dtype, rows, cols):
    """A batch without tokens still has the experts' padding rows."""
    none = torch.empty((0, cols), dtype=dtype, device="cuda")
    ids, weights, dw = (torch.empty((0, 2), dtype=t, device="cuda") for t in (I32, F32, F32))
    order = torch.empty((rows,), dtype=I32, device="cuda")
    offsets, pos = torch.empty((2,), dtype=I32, device="cuda"), torch.empty((0,), dtype=I32, device="cuda")
    so.sfc_moe_sort(ids, offsets, order, pos)
    assert (order == -1).all() and (offsets == 0).all()
    dys, full = framed(rows, cols, dtype)
    ys = torch.ones((rows, cols), dtype=dtype, device="cuda")
    for o in (order, torch.arange(rows, dtype=I32, device="cuda")):      # slots that do not exist count as none
        full.fill_(9)
        so.sfc_moe_combine_grad(none, ys, o, pos, weights, dys, dw)
        assert (dys == 0).all() and frame_is_whole(full, rows, cols)
        full.fill_(9)
        so.sfc_moe_dispatch(none, o, dys, topk=2)
        assert (dys == 0).all() and frame_is_whole(full, rows, cols)
    so.sfc_moe_combine(ys, pos, none)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 17, 31])
@pytest.mark.parametrize("cols", [1, 300, 2050])
def test_tokens_without_rows(so, dtype, rows, cols):
    """Every slot dropped: sums are 0, no row belongs to a slot."""
    T = 3
    dy = torch.ones((T, cols), dtype=dtype, device="cuda")
    pos = torch.full((2 * T,), -1, dtype=I32, device="cuda")
    order = torch.full((rows,), -1, dtype=I32, device="cuda")
    dys, full = framed(rows, cols, dtype)
    dw = torch.full((T, 2), 9.0, device="cuda")
    so.sfc_moe_combine_grad(dy, torch.ones((rows, cols), dtype=dtype, device="cuda"), order, pos, None, dys, dw)
    assert (dys == 0).all() and (dw == 0).all() and frame_is_whole(full, rows, cols)
    y, full = framed(T, cols, dtype)
    so.sfc_moe_combine(torch.ones((rows, cols), dtype=dtype, device="cuda"), pos, y)
    assert (y == 0).all() and frame_is_whole(full, T, cols)
