"""Adapters, up, with 256 rows to a workgroup at every rank: whole numbers, exact."""
import pytest
import torch

from lora_cases import TALL
from rows_cases import BF16, F32, framed, small_ints, untouched_outside
from test_gpu_lora import make_ids, same, so, up  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,rank,adapters", TALL)
@pytest.mark.parametrize("kind", ["rows", "runs"])
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_up_of_256_rows_to_a_workgroup(so, rows, cols, rank, adapters, kind, nk, dtype, pad, shift):  # noqa: F811
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
    assert same(y, want) and untouched_outside(y)
    so.sfc_lora_up(v, b, ids, base, base=base, layout=lay)
    assert same(base, want) and untouched_outside(base)
