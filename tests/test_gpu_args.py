"""The C++ argument checks of the operators' binding (_sfcargs) against what the Python code behind
them gives, and that they leave every other argument to it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U8, F32, BF16, I32 = torch.uint8, torch.float32, torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def so():
    from paper_2601_16294_amd import sfcops
    return sfcops


def slow(so, monkeypatch):
    for name in ("_rows_of", "_mx4_of", "_vector_of", "_empty_of"):
        monkeypatch.setattr(so, name, lambda *a: None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("make", [
    lambda x: x, lambda x: x[:, 3:], lambda x: x[::2], lambda x: x[:1], lambda x: x[:0], lambda x: x[:, :1], lambda x: x[:, :0],
    lambda x: x.T[:1].T])
def test_rows(so, monkeypatch, dtype, make):
    t = make(torch.zeros(6, 40, device="cuda", dtype=dtype))
    got = so._rows_of(t, -1, -1)
    assert got is not None and so._rows_of(t, *t.shape) == got and so._rows_of(t, t.shape[0] + 1, t.shape[1]) is None
    slow(so, monkeypatch)
    assert so._rows(t, "t", "test") == got


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (5, 32), (5, 100), (7, 128), (0, 64), (3, 0)])
@pytest.mark.parametrize("lead", [0, 1])
def test_mx4(so, monkeypatch, rows, cols, lead):
    q, s = so.mx4_empty(rows, cols, lead=(3,) * lead)
    got = so._mx4_of(q, s, lead, -1, -1)
    assert got is not None and so._mx4_of(q, s, lead, rows, (cols + 31) // 32) == got
    assert so._mx4_of(q, s, lead, rows + 1, (cols + 31) // 32) is None and so._mx4_of(q, s, lead, rows, 99) is None
    slow(so, monkeypatch)
    assert so._mx4(q, s, "q", "test", lead=lead) == got
    like = so.mx4_empty(rows, cols, lead=(3,) * lead)
    for a, b in zip((q, s), like):
        assert a.shape == b.shape and a.stride() == b.stride() and a.dtype == b.dtype and a.device == b.device


def test_vector(so):
    f, i = torch.zeros(6, device="cuda"), torch.zeros(2, 3, device="cuda", dtype=I32)
    assert so._vector_of(f, True, 6) == f.data_ptr() and so._vector_of(i, False, -1) == i.data_ptr()
    for bad in [(f, False, 6), (i, True, 6), (f, True, 5), (f[::2], True, 3), (f.cpu(), True, 6), (None, True, 6)]:
        assert so._vector_of(*bad) is None


class Sub(torch.Tensor):
    pass


def test_everything_else_is_left_to_python(so):
    x = torch.zeros(4, 64, device="cuda")
    for bad in [None, 3, "x", x.cpu(), x[0], x.double(), x.T, x[:, ::2], x.to_sparse(), x.as_subclass(Sub)]:
        assert so._rows_of(bad, -1, -1) is None
    q, s = so.mx4_empty(4, 96)
    pairs = [(q, None), (None, s), (q.cpu(), s), (q, s.cpu()), (q.float(), s), (q, s.int()), (q[:3], s), (q, s[:, :2]), (q[:, ::2], s),
             (q[None], s), (q, torch.zeros(4, 3, dtype=U8, device="cuda"))]      # (the last: ends inside a group of 4)
    for a, b in pairs:
        assert so._mx4_of(a, b, 0, -1, -1) is None
    # a subclass on the GPU is taken all the same, by the Python code
    so.sfc_mx4_quant(torch.zeros(4, 96, device="cuda").as_subclass(Sub), q, s)
    with pytest.raises((TypeError, RuntimeError)):
        so.mx4_empty(4, "x")
