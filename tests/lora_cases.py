"""Shapes of the low-rank adapters' calls that are taken in tiles, shared by the GPU tests and the CPU test that every kernel
is reached, and reference sums that keep infinities and NaN where the formulas have them."""
import torch

# (rows, columns, rank, adapters): down and up in tiles, every chunk count of up; the weight gradient in parts and whole, rows
# of Z or V of fewer than 8 elements too
SPECIAL = [(4100, 70, 12, 5), (2100, 1100, 40, 2), (1500, 515, 100, 2), (600, 520, 256, 4), (4500, 5, 3, 3), (4101, 64, 8, 1),
           (600, 8200, 256, 2)]


def product(v, w):
    """v (rows, rank) times w (columns, rank) transposed in 64 bits, every product formed and added by itself, so that an
    infinity or NaN reaches the sums it belongs to and no other; and the sum of the finite products' magnitudes."""
    out = torch.empty((v.shape[0], w.shape[0]), dtype=torch.float64, device=v.device)
    size = torch.empty_like(out)
    step = max(1, (1 << 26) // max(1, w.numel()))
    for i in range(0, v.shape[0], step):
        p = v[i:i + step].double()[:, None, :] * w.double()[None]
        out[i:i + step] = p.sum(-1)
        size[i:i + step] = torch.where(torch.isfinite(p), p.abs(), 0.0).sum(-1)
    return out, size


def special(t, places, values, seed):
    """Puts the values, in turn, at random places of t."""
    g = torch.Generator().manual_seed(seed)
    for i in range(places):
        at = tuple(int(torch.randint(0, n, (1,), generator=g)) for n in t.shape)
        t[at] = values[i % len(values)]


def agrees(got, want, bound):
    """NaN where the formula has NaN, the same infinities, and finite values within `bound`."""
    g = got.double()
    fine = torch.where(torch.isfinite(want), (g - want).abs() <= bound, (g == want) | (torch.isnan(g) & torch.isnan(want)))
    return bool(fine.all())

# (rows, columns, rank, adapters) that up takes with 256 rows to a workgroup, for every chunk count
TALL = [(8300, 4003, 24, 3), (8200, 4100, 40, 4), (8300, 2050, 100, 3), (8300, 1030, 256, 2), (8200, 1040, 129, 3)]
