"""Whole numbers that do not fit the C ABI's ints are refused by the binding: cut to 32 bits, 2^32 + 2
choices would pass for 2.  No GPU is needed."""
import pytest
import torch

from paper_2601_16294_amd import sfcops as so

I32 = torch.int32


@pytest.fixture
def calls(monkeypatch):
    """Host tensors pass the device check; what reaches the library is kept."""
    got = []
    monkeypatch.setattr(so, "_tensor", lambda t, name, what: None)
    monkeypatch.setattr(so, "_stream", lambda s: None)

    class Lib:
        def __getattr__(self, name):
            return lambda *a: got.append((name, a)) or 0
    monkeypatch.setattr(so, "lib", Lib())
    return got


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def long(n):
    """n whole numbers that take no memory, contiguous as far as the binding asks."""
    return torch.zeros(1, dtype=I32).expand(n)


BIG = (1 << 32) + 2


@pytest.mark.parametrize("f", [
    lambda: so.sfc_mx4_quant(t(4, 128), *so.mx4_empty(8, 128, device="cpu"), order=t(8, dtype=I32), topk=BIG),
    lambda: so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(8, 32), topk=BIG),
    lambda: so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(8, 32), topk=1 << 31),
    lambda: so.sfc_moe_sort(t(4, 2, dtype=I32), t(9, dtype=I32), t(8, dtype=I32), t(8, dtype=I32), align=BIG),
    lambda: so.sfc_moe_sort(t(4, 2, dtype=I32), t(9, dtype=I32), t(8, dtype=I32), t(8, dtype=I32), align=-BIG),
])
def test_numbers(calls, f):
    with pytest.raises(ValueError, match=r"2\^31"):
        f()
    assert calls == []


def test_counts_of_elements(calls, monkeypatch):
    """Counts that come from a tensor's shape (a contiguous one of so many elements would be 17 GB)."""
    monkeypatch.setattr(so, "_ints", lambda t, name, what, count: 0)
    for f in (lambda: so.sfc_moe_sort(t(4, 2, dtype=I32), long(BIG + 1), t(8, dtype=I32), t(8, dtype=I32)),
              lambda: so.sfc_moe_combine(t(8, 32), long(BIG), t(1, 32)),
              lambda: so.sfc_moe_wgrad_mx4_ex(*so.mx4_empty(4, 128, device="cpu"), *so.mx4_empty(8, 128, device="cpu"), long(BIG + 1),
                                              torch.zeros(1, 1, 1).expand(BIG, 4, 8))):
        with pytest.raises(ValueError, match=r"2\^31"):
            f()
    assert calls == []


def test_the_largest_that_fits_reaches_the_library(calls):
    so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(8, 32), topk=(1 << 31) - 1)
    so.sfc_moe_sort(t(4, 2, dtype=I32), t(9, dtype=I32), t(8, dtype=I32), t(8, dtype=I32), align=1 << 20)
    assert calls[0][1][3] == (1 << 31) - 1 and calls[1][1][1:3] == (8, 1 << 20)
