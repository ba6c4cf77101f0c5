"""Whole numbers that do not fit the C ABI's ints are refused by the workspace sizes of the adapters: cut to 32 bits,
2^32 + 2 adapters would pass for 2, and rows past 2^64 for few.  No GPU is needed."""
import pytest

from paper_2601_16294_amd import sfcops as so


@pytest.mark.parametrize("f", [so.sfc_lora_down_ws_size, so.sfc_lora_wgrad_ws_size])
@pytest.mark.parametrize("at", [0, 1, 2, 3])
@pytest.mark.parametrize("n", [(1 << 32) + 64, (1 << 64) + 64, -(1 << 64) + 64])
def test_sizes(f, at, n):
    sizes = [4096, 4096, 16, 8]
    sizes[at] = n
    if at < 3 and abs(n) < 1 << 63:
        assert f(*sizes) == 0                        # (the library sees the number itself, which no call takes)
    else:
        with pytest.raises(ValueError, match=r"2\^31"):
            f(*sizes)


@pytest.mark.parametrize("f", [so.sfc_lora_down_ws_size, so.sfc_lora_wgrad_ws_size])
def test_what_fits_reaches_the_library(f, monkeypatch):
    got = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: got.append((name, a)) or 48
    monkeypatch.setattr(so, "lib", Lib())
    assert f((1 << 31) - 1, 5, 0, (1 << 31) - 1) == 48
    assert got == [(f.__name__, ((1 << 31) - 1, 5, 0, (1 << 31) - 1))]
