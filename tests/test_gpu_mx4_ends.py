"""4-bit operands whose scales end with their allocation, in block shapes that end in one row:
loads of scales run ahead of the range of K, and no byte past the last row's may be read.
Products are exact (see test_gpu_mx4), so rows at the end are compared bit by bit."""
import numpy as np
import pytest
import torch

from oracle import mx4

pytestmark = pytest.mark.gpu
PAGE = 2 << 20                       # allocations from 10 MB on are whole multiples of it


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def at_the_end(rows, K, seed):
    """(codes, scales) of rows x K random values, the scales at the end of an allocation."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks, padded = K // 32, (K // 32 + 3) // 4 * 4
    q = torch.randint(0, 256, (rows, 16 * blocks), generator=g, device="cuda", dtype=torch.uint8)
    size = max(-(-rows * padded // PAGE) * PAGE, 6 * PAGE)
    torch.cuda.empty_cache()
    buf = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    s = buf[size - rows * padded:].view(rows, padded)
    s[:, :blocks] = torch.randint(127, 129, (rows, blocks), generator=g, device="cuda", dtype=torch.uint8)
    return q, s[:, :blocks]


def values(q, s):
    return torch.from_numpy(mx4.values(mx4.unpack(q.cpu().numpy()), s.cpu().numpy())).cuda()


# |a b| <= 36 * 4 in steps of 1/4: the sums are exact
@pytest.mark.parametrize("rows,K", [(256 * 12287 + 1, 128), (256 * 383 + 1, 4096), (128 * 700 + 1, 4000), (256 * 300 + 3, 32)])
@pytest.mark.parametrize("side", ["A", "B"])
def test_products(so, rows, K, side):
    big, small = at_the_end(rows, K, 1), at_the_end(70, K, 2)
    out = (rows, 70) if side == "A" else (70, rows)
    C = torch.empty(out, dtype=torch.float32, device="cuda")
    so.sfc_gemm_mx4_ex(*(big + small if side == "A" else small + big), C)
    C = C if side == "A" else C.t()
    for part in (slice(0, 300), slice(rows - 300, rows)):
        want = values(big[0][part], big[1][part]) @ values(*small).t()
        assert torch.equal(C[part].double(), want)


@pytest.mark.parametrize("M,N,K", [(1, 70, 4000), (16, 1000, 128), (17, 70, 32), (33, 130, 2080)])
def test_few_rows(so, M, N, K):
    a, b = at_the_end(M, K, 3), at_the_end(N, K, 4)
    C = torch.empty((M, N), dtype=torch.float32, device="cuda")
    so.sfc_gemm_mx4_ex(*a, *b, C)
    assert torch.equal(C.double(), values(*a) @ values(*b).t())


@pytest.mark.parametrize("K", [32, 160, 4128])
def test_experts(so, K):
    rows, N, E = 385, 129, 3
    A, B = at_the_end(rows, K, 5), at_the_end(E * N, K, 6)
    offsets = torch.tensor([0, 129, 129, 385], dtype=torch.int32, device="cuda")
    C = torch.empty((rows, N), dtype=torch.float32, device="cuda")
    Bs = B[1].as_strided((E, N, K // 32), (N * B[1].stride(0), B[1].stride(0), 1), B[1].storage_offset())
    so.sfc_moe_gemm_mx4_ex(*A, B[0].view(E, N, -1), Bs, offsets, C)
    a, b = values(*A), values(*B).view(E, N, K)
    for e, (lo, hi) in enumerate(((0, 129), (129, 129), (129, 385))):
        assert torch.equal(C[lo:hi].double(), a[lo:hi] @ b[e].t())


@pytest.mark.parametrize("starts", [[0, 32], [0, 96, 96, 1312], [0, 4096, 4224]])
def test_weight_gradients(so, starts):
    M, N, K = 257, 129, starts[-1]
    A, B = at_the_end(M, K, 7), at_the_end(N, K, 8)
    C = torch.empty((len(starts) - 1, M, N), dtype=torch.float32, device="cuda")
    so.sfc_moe_wgrad_mx4_ex(*A, *B, torch.tensor(starts, dtype=torch.int32, device="cuda"), C)
    a, b = values(*A), values(*B)
    for e, (lo, hi) in enumerate(zip(starts[:-1], starts[1:])):
        assert torch.equal(C[e].double(), a[:, lo:hi] @ b[:, lo:hi].t())
