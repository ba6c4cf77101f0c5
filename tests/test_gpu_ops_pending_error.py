"""An error that an earlier HIP call of the program left behind (here: a device number that does not
exist) is not a call's own: the operators launch, succeed and give their results."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def calls(so):
    """name -> (call, its outputs)"""
    x = torch.randn((40, 160), device="cuda").to(BF16)
    q, qt, w = so.mx4_empty(40, 160), so.mx4_empty(160, 40), so.mx4_empty(64, 160)
    so.sfc_mx4_quant(x, *q)
    so.sfc_mx4_quant(torch.randn((64, 160), device="cuda"), *w)
    out = lambda *shape, dtype=F32: torch.zeros(shape, dtype=dtype, device="cuda")
    q2, y, c, z = so.mx4_empty(40, 160), out(40, 160), out(40, 64), out(40, 64)
    for t in (*q2, *qt):
        t.zero_()
    ids = torch.arange(10000, device="cuda", dtype=I32) % 8
    offsets, order, pos = out(9, dtype=I32), out(10000, dtype=I32), out(10000, dtype=I32)
    few, fpos = torch.arange(40, device="cuda", dtype=I32), torch.arange(40, device="cuda", dtype=I32)
    xs, ys, dys, dw = out(40, 160, dtype=BF16), out(40, 160, dtype=BF16), out(40, 160, dtype=BF16), out(40, 1)
    e, we, off = out(40, 64), tuple(t[None] for t in w), torch.tensor([0, 40], device="cuda", dtype=I32)
    g, off160 = out(1, 64, 64), torch.tensor([0, 160], device="cuda", dtype=I32)
    return {
        "quant": (lambda: so.sfc_mx4_quant(x, *q2), q2), "quant columns": (lambda: so.sfc_mx4_quant(x, None, None, *qt), qt),
        "dequant": (lambda: so.sfc_mx4_dequant(*q, y), (y,)), "product": (lambda: so.sfc_gemm_mx4_ex(*q, *w, c), (c,)),
        "linear": (lambda: so.sfc_mx4_linear(x, *w, z), (z,)), "sort": (lambda: so.sfc_moe_sort(ids, offsets, order, pos), (offsets, order, pos)),
        "dispatch": (lambda: so.sfc_moe_dispatch(x, few, xs), (xs,)), "combine": (lambda: so.sfc_moe_combine(x, fpos, ys), (ys,)),
        "gradient": (lambda: so.sfc_moe_combine_grad(x, x, few, fpos, None, dys, dw), (dys, dw)),
        "experts": (lambda: so.sfc_moe_gemm_mx4_ex(*q, *we, off, e), (e,)),
        "weight gradient": (lambda: so.sfc_moe_wgrad_mx4_ex(*w, *w, off160, g), (g,)),
    }


@pytest.mark.parametrize("name", ["quant", "quant columns", "dequant", "product", "linear", "sort", "dispatch", "combine", "gradient", "experts",
                                  "weight gradient"])
def test_it_is_left_alone(so, name):
    call, outputs = calls(so)[name]
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    for t in outputs:
        t.zero_()
    torch.cuda.synchronize()
    hip = so.lib                                     # (the library's own HIP runtime)
    hip.hipSetDevice.argtypes = [ctypes.c_int]
    assert hip.hipSetDevice(1000) != 0
    try:
        call()
    finally:
        hip.hipGetLastError()                        # torch would report it as one of its own launches'
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, want))


# (grids that no other test has: the curve table is made, and the layers summed, behind the error)
@pytest.mark.parametrize("entry", ["mx4", "bf16"])
@pytest.mark.parametrize("N", [1290, 1291])
def test_layers_on_a_new_grid(so, entry, N):
    from paper_2601_16294_amd import sfcgemm as sg
    M, K = 390 if entry == "mx4" else 3000, 8192
    a, b = torch.randn((M, K), device="cuda").to(BF16), torch.randn((K, N), device="cuda").to(BF16)
    aq, bq = so.mx4_empty(M, K), so.mx4_empty(N, K)
    so.sfc_mx4_quant(a, *aq)
    so.sfc_mx4_quant(b, None, None, *bq)
    got, want = (torch.zeros((M, N), device="cuda") for _ in range(2))
    f = (lambda c: so.sfc_gemm_mx4_ex(*aq, *bq, c)) if entry == "mx4" else (lambda c: sg.sfc_gemm_ex(a, b, c, ca_layers=3, tile="128x128"))
    torch.cuda.synchronize()
    so.lib.hipSetDevice.argtypes = [ctypes.c_int]
    assert so.lib.hipSetDevice(1000) != 0
    try:
        f(got)
    finally:
        so.lib.hipGetLastError()
    f(want)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and want.abs().max() > 0
