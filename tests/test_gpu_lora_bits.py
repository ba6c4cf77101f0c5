"""What the adapters' calls keep of V in tiles: all of its 24 bits in fp32 results and gradients.  Where one product of a sum is not
0, the result has to be that product."""
import pytest
import torch

from lora_cases import SPECIAL, TALL
from rows_cases import BF16
from test_gpu_lora import so  # noqa: F401

pytestmark = pytest.mark.gpu


def odd_24(shape, seed):
    """Odd whole numbers of 24 bits, of both signs: no fewer bits hold them."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(1 << 22, 1 << 23, shape, generator=g) * 2 + 1
    return (t * (torch.randint(0, 2, shape, generator=g) * 2 - 1)).float().cuda()


def one_a_row(rows, rank, values):
    """values (rows) at one rank of every row, zeros else."""
    v = torch.zeros((rows, rank), device="cuda")
    at = torch.arange(rows, device="cuda") * 7 % rank
    v[torch.arange(rows, device="cuda"), at] = values
    return v, at


@pytest.mark.parametrize("rows,cols,rank,n", SPECIAL + TALL)
@pytest.mark.parametrize("nk", [True, False])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -130, 2.0 ** 100])
def test_up_has_every_bit_of_v(so, rows, cols, rank, n, nk, scale):  # noqa: F811
    """fp32 results of weights +-1 and of powers of two, of V with 24 bits; at 2^-130 times that what reaches below 2^-134 may
    be lost (of V: of results with weights of up to 4, 2^-132)."""
    ids = (torch.arange(rows, device="cuda") * 5 % (n + 1)).to(torch.int32)
    v, at = one_a_row(rows, rank, odd_24((rows,), 1) * scale)
    g = torch.Generator().manual_seed(2)
    b = torch.exp2(torch.randint(-2, 3, (n, cols, rank), generator=g).float()) * (torch.randint(0, 2, (n, cols, rank), generator=g) * 2 - 1)
    b = b.cuda().to(BF16)
    y = torch.full((rows, cols), 5.0, device="cuda")
    so.sfc_lora_up(v, b if nk else b.transpose(1, 2).contiguous(), ids, y, layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    live = ids < n
    want = torch.zeros_like(y)
    own = v[torch.arange(rows, device="cuda"), at]
    for i in range(n):
        t = torch.nonzero(ids == i)[:, 0]
        want[t] = own[t, None] * b[i].float().t()[at[t]]
    assert not y[~live].any()
    if scale < 1:
        assert ((y.double() - want.double()).abs() <= 2.0 ** -132).all()
    else:
        assert torch.equal(y, want)


@pytest.mark.parametrize("rows,cols,rank,n", [(40, 70, 12, 40), (300, 515, 100, 300), (90, 520, 256, 90), (30, 5, 3, 30), (4096, 64, 8, 1)])
@pytest.mark.parametrize("nk", [True, False])
def test_gradient_has_every_bit_of_v(so, rows, cols, rank, n, nk):  # noqa: F811
    """A row that is not 0 for every adapter, Z of powers of two."""
    ids = (torch.arange(rows, device="cuda") % n).to(torch.int32)
    g = torch.Generator().manual_seed(3)
    z = torch.exp2(torch.randint(-3, 4, (rows, cols), generator=g).float()).cuda().to(BF16)
    v = odd_24((rows, rank), 4)
    v[n:] = 0
    out = torch.full((n, cols, rank) if nk else (n, rank, cols), 5.0, device="cuda")
    so.sfc_lora_wgrad(z, v, ids, out, layout=so.SFC_B_NK if nk else so.SFC_B_KN)
    want = z[:n].float()[:, :, None] * v[:n, None, :]
    assert torch.equal(out if nk else out.transpose(1, 2), want)
