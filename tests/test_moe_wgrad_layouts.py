"""Layouts of the experts' weight gradients: one matrix behind the other, or the experts' rows in turn."""
import pytest
import torch

from paper_2601_16294_amd import sfcops as so
from test_ops_refusals import DEPTH, WGOOD, call

lib = so.lib


# (M = N = 64, 4 experts; a C of null passes the checks of strides only if they are good, and fails after them)
@pytest.mark.parametrize("kw,code", [
    (dict(ldc=256, sc=64), 0), (dict(ldc=300, sc=70), 0), (dict(ldc=64, sc=4096), 0), (dict(ldc=100, sc=6364), 0), (dict(E=1, sc=0), 0),
    (dict(M=1, ldc=64, sc=64), 0),
    (dict(ldc=255, sc=64), -1), (dict(ldc=256, sc=63), -1), (dict(ldc=256, sc=0), -1), (dict(ldc=256, sc=65), -1),
    (dict(ldc=100, sc=6363), -1), (dict(M=1, ldc=64, sc=63), -1)])
def test_strides(kw, code):
    # good strides get as far as the check behind them: offsets
    assert call(lib.sfc_moe_wgrad_mx4_ex, DEPTH, WGOOD, dict(kw, offsets=None)) == -1
    text = lib.sfc_last_error().decode()
    assert ("offsets" in text) == (code == 0) and ("overlap" in text) == (code != 0)


@pytest.mark.gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_rows_in_turn(out):
    from test_gpu_mx4 import check, operand
    starts, M, N = [0, 96, 96, 800, 1024], 129, 257
    A, As, a = operand(M, 1024, 3)
    B, Bs, b = operand(N, 1024, 4)
    C = torch.full((M, 4, N + 3), 99.0, dtype=out, device="cuda")
    so.sfc_moe_wgrad_mx4_ex(A, As, B, Bs, torch.tensor(starts, dtype=torch.int32, device="cuda"), C[:, :, 1:1 + N].transpose(0, 1))
    assert (C[:, :, 0] == 99).all() and (C[:, :, 1 + N:] == 99).all()
    for e in range(4):
        check(C[:, e, 1:1 + N], a[:, starts[e]:starts[e + 1]], b[:, starts[e]:starts[e + 1]], 1024, True)
