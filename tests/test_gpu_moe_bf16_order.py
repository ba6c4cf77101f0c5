"""Experts' products that gather their rows through a sort order, with bf16 results, on blocks of every size.  Whole numbers, whose
fp32 sums are exact: a bf16 result is their rounding, bit for bit."""
import numpy as np
import pytest
import torch

from rows_cases import BF16, EXPERTS, framed, offsets_of, small_ints, untouched_outside
from test_gpu_moe_bf16 import product, same, so  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,N,K", [e for e in EXPERTS if sum(e[0]) > 0])
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("topk", [1, 3])
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 1)])
def test_bf16_product_of_rows_through_an_order(so, counts, N, K, nk, topk, pad, shift):  # noqa: F811
    rows, E, tokens = sum(counts), len(counts), 37
    rng = np.random.default_rng(rows + N)
    order = rng.integers(0, tokens * topk, rows + 2).astype(np.int32)
    order[rng.random(rows + 2) < 0.2] = rng.choice([-1, -(1 << 31), tokens * topk, (1 << 31) - 1])
    x = small_ints((tokens, K), 3, pad, shift)
    b = small_ints((E, N, K) if nk else (E, K, N), 4, pad, shift)
    c = framed((rows + 2, N), BF16, pad, shift)
    so.sfc_moe_gemm_ex(x, b, offsets_of(counts), c, order=torch.from_numpy(order).cuda(), topk=topk,
                       layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    src = torch.from_numpy(np.where((order >= 0) & (order // topk < tokens), order // topk, tokens).astype(np.int64)).cuda()
    a = torch.cat([x, torch.zeros((1, K), dtype=BF16, device="cuda")])[src[:rows]]
    assert same(c[:rows], product(a, b, counts, nk))
    assert (c[rows:] == 0).all() and untouched_outside(c)
