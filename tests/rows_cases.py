"""Shapes of the bf16 experts' products, shared by the GPU tests and the routing test (no GPU), so that
no kernel goes untested when a rule moves, and helpers to lay them out."""
import numpy as np
import torch

BF16, F32 = torch.bfloat16, torch.float32

# (rows of every expert, N, K)
EXPERTS = [
    ([1], 1, 1), ([1], 16, 32), ([0, 0, 3], 100, 96), ([2, 1, 0, 5, 16, 17, 0, 1], 333, 545), ([40, 0, 1, 70], 64, 1024),
    ([20, 30, 33], 70, 4129), ([70, 200, 0, 129], 200, 63), ([128, 128, 256], 257, 512), ([1, 2] * 32, 601, 288),
    ([0, 0, 0, 0], 70, 64), ([5, 300], 5, 200), ([9, 130], 3, 7), ([0, 2000, 1], 4096, 129), ([3, 2], 130, 0),
    ([1000, 3, 0, 1500], 7000, 1032), ([700, 0, 1111, 1256, 257, 1000, 511, 768], 4100, 1031), ([4096], 4096, 264),
    ([3000, 5000], 8200, 70),
]

# (rows of every expert, N, K) with rows of 16-byte pieces: the kernels that stream the weights
FEW = [
    ([1], 1, 8), ([0, 3, 0, 8], 130, 264), ([1, 0, 16, 17, 5, 1, 0, 0], 600, 520), ([8] * 3, 100, 4104), ([24], 333, 1096), ([20], 32, 40),
    ([32], 1000, 2056), ([33], 95, 4096), ([40, 0, 24], 257, 512), ([64], 4096, 1544), ([1, 50], 64, 64), ([0, 0], 40, 64),
]

# (rows of every expert, M, N)
DEPTHS = [
    ([1], 1, 1), ([32], 16, 16), ([0, 0, 64, 1, 31], 130, 70), ([33, 127, 2000], 200, 300), ([96, 0, 704, 200], 129, 257),
    ([4096], 100, 60), ([3, 66, 129], 5, 3), ([200, 7], 1, 9), ([65, 64, 63, 0, 1], 256, 256), ([0, 0], 33, 20),
    ([300, 1, 0, 411], 2040, 2047), ([1000, 640], 4096, 1600), ([200, 100], 3100, 3000),
    ([1500, 1100], 5000, 3403),
]


def offsets_of(counts):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()


def framed(shape, dtype, ld_pad=0, shift=0, gap=0):
    """A tensor (rows, cols) or (n, rows, cols) inside memory that is NaN all around it: `ld_pad` elements behind
    every row, `shift` elements off the start, `gap` elements between matrices."""
    *lead, rows, cols = shape
    n, ld = (lead[0] if lead else 1), cols + ld_pad
    stride = rows * ld + gap
    flat = torch.full((shift + n * stride + 64,), float("nan"), dtype=dtype, device="cuda")
    t = torch.as_strided(flat, (n, rows, cols), (stride, ld, 1), shift)
    return t if lead else t[0]


def small_ints(shape, seed, ld_pad=0, shift=0, gap=0, most=8):
    """Whole numbers of up to `most` in magnitude as bf16: sums of 2^24 / most^2 products are exact in fp32."""
    g = torch.Generator().manual_seed(seed)
    t = framed(shape, BF16, ld_pad, shift, gap)
    t.copy_(torch.randint(-most, most + 1, tuple(shape), generator=g).to(BF16).cuda())
    return t


def normals(shape, seed, scale=1.0, ld_pad=0, shift=0, gap=0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    t = framed(shape, dtype, ld_pad, shift, gap)
    t.copy_((torch.randn(tuple(shape), generator=g) * scale).to(dtype).cuda())
    return t


def untouched_outside(t):
    """Whether all memory of a framed tensor's buffer outside of it is still NaN."""
    flat = torch.as_strided(t, (t.untyped_storage().nbytes() // t.element_size(),), (1,), 0).clone()
    mask = torch.ones(flat.numel(), dtype=torch.bool, device=t.device)
    torch.as_strided(mask, t.shape, t.stride(), t.storage_offset()).fill_(False)
    return bool(torch.isnan(flat[mask]).all())


def close(got, want, size, terms, dtype):
    """|got - want| within what fp32 sums of `terms` exact products of magnitudes that add up to `size` and one rounding
    of the result to `dtype` may be off."""
    bound = terms * 2.0 ** -23 * size
    if dtype == BF16:
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    return bool(((got.double() - want).abs() <= bound).all())
