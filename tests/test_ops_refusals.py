"""The 4-bit and expert operators refuse bad arguments before any HIP call: wrong sizes, strides,
alignment, types and devices, at the C ABI and at the Python binding.  No GPU is needed."""
import pytest
import torch

from paper_2601_16294_amd import sfcops as so

lib = so.lib
F32, BF16 = 0, 1
A, S, B, T, C, O = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000


def call(fn, order, good, kw):
    a = dict(good)
    a.update(kw)
    return fn(*[a[k] for k in order.split()])


QUANT = "rows cols X ldx type order x_rows topk Q ldq S lds Qt ldqt St ldst stream"
QGOOD = dict(rows=64, cols=96, X=A, ldx=96, type=BF16, order=None, x_rows=0, topk=0, Q=B, ldq=48, S=S, lds=4, Qt=C, ldqt=32,
             St=T, ldst=4, stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(cols=-1), -1), (dict(X=None), -1), (dict(ldx=95), -1), (dict(type=2), -1),
    (dict(Q=None), -1), (dict(S=None), -1), (dict(Qt=None), -1), (dict(Q=None, S=None, Qt=None, St=None), -1),
    (dict(ldq=32), -1), (dict(lds=0), -1), (dict(ldqt=16), -1), (dict(ldst=0), -1),
    (dict(ldq=56), -2), (dict(Q=B + 8), -2), (dict(S=S + 2), -2), (dict(lds=6), -2), (dict(X=A + 1), -2),
    (dict(type=F32, X=A + 2), -2), (dict(rows=1 << 31), -2), (dict(ldq=1 << 22), -2),
    (dict(order=O, x_rows=4, topk=0), -1), (dict(order=O + 2, x_rows=4, topk=1), -2), (dict(order=O, x_rows=-1, topk=1), -1)])
def test_quant(kw, code):
    assert call(lib.sfc_mx4_quant, QUANT, QGOOD, kw) == code
    assert "" != so.SfcError(code, "x").args[0]


def test_nothing_to_do_is_success():
    assert call(lib.sfc_mx4_quant, QUANT, QGOOD, dict(rows=0, X=None, Q=None, S=None, Qt=None, St=None)) == 0
    assert call(lib.sfc_mx4_dequant, DEQUANT, DGOOD, dict(cols=0, Q=None, S=None, Y=None)) == 0
    assert call(lib.sfc_gemm_mx4_ex, GEMM, GGOOD, dict(M=0, A=None, As=None, C=None)) == 0
    assert call(lib.sfc_mx4_linear, LINEAR, LGOOD, dict(N=0, W=None, Ws=None, Y=None)) == 0
    assert call(lib.sfc_moe_gemm_mx4_ex, EXPERTS, EGOOD, dict(rows=0, A=None, C=None)) == 0
    assert call(lib.sfc_moe_wgrad_mx4_ex, DEPTH, WGOOD, dict(M=0, A=None, C=None)) == 0
    assert call(lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(rows=0, Xs=None, order=None)) == 0
    assert call(lib.sfc_moe_combine, COMBINE, CGOOD, dict(tokens=0, Y=None, pos=None)) == 0
    assert call(lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(tokens=0, rows=0, order=None, pos=None, dW=None)) == 0


DEQUANT = "rows cols Q ldq S lds Y ldy type stream"
DGOOD = dict(rows=8, cols=96, Q=A, ldq=48, S=S, lds=4, Y=C, ldy=96, type=BF16, stream=None)


@pytest.mark.parametrize("kw,code", [(dict(Q=None), -1), (dict(Y=None), -1), (dict(ldy=95), -1), (dict(ldq=32), -1),
                                     (dict(type=5), -1), (dict(Y=C + 1), -2), (dict(lds=5), -2)])
def test_dequant(kw, code):
    assert call(lib.sfc_mx4_dequant, DEQUANT, DGOOD, kw) == code


GEMM = "M N K A lda As ldas B ldb Bs ldbs C ldc out stream"
GGOOD = dict(M=64, N=64, K=128, A=A, lda=64, As=S, ldas=4, B=B, ldb=64, Bs=T, ldbs=4, C=C, ldc=64, out=F32, stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), -1), (dict(K=100), -1), (dict(K=-32), -1), (dict(A=None), -1), (dict(As=None), -1), (dict(B=None), -1),
    (dict(Bs=None), -1), (dict(C=None), -1), (dict(lda=48), -1), (dict(ldb=48), -1), (dict(ldc=63), -1), (dict(out=2), -1),
    (dict(A=A + 8), -2), (dict(lda=72), -2), (dict(As=S + 1), -2), (dict(ldbs=7), -2), (dict(C=C + 2), -2),
    (dict(M=1 << 31), -2), (dict(K=1 << 24, lda=1 << 23, ldb=1 << 23, ldas=1 << 19, ldbs=1 << 19), -2),
    (dict(M=(1 << 31) - 1, N=(1 << 31) - 1, ldc=(1 << 31) - 1), -2)])
def test_gemm(kw, code):
    assert call(lib.sfc_gemm_mx4_ex, GEMM, GGOOD, kw) == code


LINEAR = "M N K X ldx type W ldw Ws ldws Y ldy out stream"
LGOOD = dict(M=64, N=64, K=100, X=A, ldx=100, type=BF16, W=B, ldw=64, Ws=T, ldws=4, Y=C, ldy=64, out=F32, stream=None)


@pytest.mark.parametrize("kw,code", [(dict(K=-1), -1), (dict(X=None), -1), (dict(ldx=99), -1), (dict(type=3), -1),
                                     (dict(ldw=48), -1), (dict(W=None), -1), (dict(Y=None), -1), (dict(ldy=1), -1),
                                     (dict(X=A + 1), -2), (dict(W=B + 4), -2), (dict(Y=C + 1), -2)])
def test_linear(kw, code):
    assert call(lib.sfc_mx4_linear, LINEAR, LGOOD, kw) == code


EXPERTS = "rows N K E A lda As ldas B ldb sb Bs ldbs ss offsets C ldc out stream"
EGOOD = dict(rows=64, N=64, K=128, E=4, A=A, lda=64, As=S, ldas=4, B=B, ldb=64, sb=4096, Bs=T, ldbs=4, ss=256, offsets=O, C=C,
             ldc=64, out=BF16, stream=None)


@pytest.mark.parametrize("kw,code", [(dict(E=0), -1), (dict(E=1025), -2), (dict(K=33), -1), (dict(offsets=None), -1),
                                     (dict(sb=-16), -1), (dict(sb=4100), -2), (dict(ss=255), -2), (dict(B=None), -1),
                                     (dict(C=None), -1), (dict(ldc=10), -1), (dict(offsets=O + 1), -2), (dict(out=9), -1)])
def test_experts(kw, code):
    assert call(lib.sfc_moe_gemm_mx4_ex, EXPERTS, EGOOD, kw) == code


DEPTH = "M N rows E A lda As ldas B ldb Bs ldbs offsets C ldc sc out stream"
WGOOD = dict(M=64, N=64, rows=128, E=4, A=A, lda=64, As=S, ldas=4, B=B, ldb=64, Bs=T, ldbs=4, offsets=O, C=C, ldc=64, sc=4096,
             out=F32, stream=None)


@pytest.mark.parametrize("kw,code", [(dict(E=0), -1), (dict(E=2000), -2), (dict(rows=-1), -1), (dict(lda=48), -1),
                                     (dict(sc=4095), -1), (dict(sc=-1), -1), (dict(offsets=None), -1), (dict(A=A + 4), -2),
                                     (dict(out=-1), -1)])
def test_depth(kw, code):
    assert call(lib.sfc_moe_wgrad_mx4_ex, DEPTH, WGOOD, kw) == code


SORT = "slots E align ids rows offsets order pos ws wsb stream"
SGOOD = dict(slots=100, E=8, align=4, ids=A, rows=124, offsets=B, order=C, pos=T, ws=None, wsb=0, stream=None)


@pytest.mark.parametrize("kw,code", [(dict(slots=-1), -1), (dict(E=0), -1), (dict(E=1025), -2), (dict(align=0), -1),
                                     (dict(align=(1 << 20) + 1), -2), (dict(rows=123), -1), (dict(ids=None), -1),
                                     (dict(offsets=None), -1), (dict(order=None), -1), (dict(pos=None), -1), (dict(pos=T + 2), -2),
                                     (dict(slots=5000, rows=5024, ws=O, wsb=63), -3), (dict(slots=5000, rows=5024, ws=O + 1, wsb=64), -2),
                                     (dict(slots=(1 << 31) - 10, rows=(1 << 31) - 1, align=32), -2)])
def test_sort(kw, code):
    assert call(lib.sfc_moe_sort, SORT, SGOOD, kw) == code


def test_sort_workspace_size():
    assert lib.sfc_moe_sort_ws_size(4096, 8) == 0 and lib.sfc_moe_sort_ws_size(4097, 8) == 64
    assert lib.sfc_moe_sort_ws_size(-1, 8) == 0 and lib.sfc_moe_sort_ws_size(5000, 0) == 0


DISPATCH = "rows cols tokens topk X ldx type order weights Xs ldxs stream"
XGOOD = dict(rows=8, cols=32, tokens=4, topk=2, X=A, ldx=32, type=BF16, order=O, weights=None, Xs=C, ldxs=32, stream=None)
COMBINE = "tokens cols rows topk Ys ldys type pos weights Y ldy stream"
CGOOD = dict(tokens=4, cols=32, rows=8, topk=2, Ys=A, ldys=32, type=F32, pos=O, weights=B, Y=C, ldy=32, stream=None)
GRAD = "tokens cols rows topk dY lddy Ys ldys type order pos weights dYs lddys dW stream"
BGOOD = dict(tokens=4, cols=32, rows=8, topk=2, dY=A, lddy=32, Ys=S, ldys=32, type=F32, order=O, pos=T, weights=None, dYs=C,
             lddys=32, dW=B, stream=None)


@pytest.mark.parametrize("fn,order,good,kw,code", [
    (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(X=None), -1), (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(order=None), -1),
    (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(topk=0), -1), (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(ldxs=31), -1),
    (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(weights=B + 1), -2), (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(type=7), -1),
    (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(Xs=C + 1), -2), (lib.sfc_moe_dispatch, DISPATCH, XGOOD, dict(tokens=1 << 30, topk=2), -2),
    (lib.sfc_moe_combine, COMBINE, CGOOD, dict(Ys=None), -1), (lib.sfc_moe_combine, COMBINE, CGOOD, dict(pos=None), -1),
    (lib.sfc_moe_combine, COMBINE, CGOOD, dict(ldy=1), -1), (lib.sfc_moe_combine, COMBINE, CGOOD, dict(Y=C + 2), -2),
    (lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(dY=None), -1), (lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(dW=None), -1),
    (lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(order=None), -1), (lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(dYs=None), -1),
    (lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(lddys=31), -1), (lib.sfc_moe_combine_grad, GRAD, BGOOD, dict(rows=-1), -1)])
def test_rows(fn, order, good, kw, code):
    assert call(fn, order, good, kw) == code


# ---- the binding: host tensors, wrong types and shapes never reach the library -------------------


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


I32 = torch.int32


@pytest.mark.parametrize("f", [
    lambda: so.sfc_mx4_quant(t(4, 32), u8(4, 16), u8(4, 1)),
    lambda: so.sfc_mx4_dequant(u8(4, 16), u8(4, 1), t(4, 32)),
    lambda: so.sfc_gemm_mx4_ex(u8(4, 16), u8(4, 1), u8(8, 16), u8(8, 1), t(4, 8)),
    lambda: so.sfc_mx4_linear(t(4, 32), u8(8, 16), u8(8, 1), t(4, 8)),
    lambda: so.sfc_moe_sort(t(4, 2, dtype=I32), t(9, dtype=I32), t(8, dtype=I32), t(8, dtype=I32)),
    lambda: so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(8, 32), topk=2),
    lambda: so.sfc_moe_combine(t(8, 32), t(8, dtype=I32), t(4, 32)),
    lambda: so.sfc_moe_combine_grad(t(4, 32), t(8, 32), t(8, dtype=I32), t(8, dtype=I32), None, t(8, 32), t(4, 2, dtype=torch.float32)),
    lambda: so.sfc_moe_gemm_mx4_ex(u8(4, 16), u8(4, 1), u8(2, 8, 16), u8(2, 8, 1), t(3, dtype=I32), t(4, 8)),
    lambda: so.sfc_moe_wgrad_mx4_ex(u8(4, 16), u8(4, 1), u8(8, 16), u8(8, 1), t(3, dtype=I32), t(2, 4, 8, dtype=torch.float32)),
])
def test_host_tensors_raise(f):
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        f()


def test_non_tensors_raise():
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        so.sfc_mx4_quant([1.0], u8(4, 16), u8(4, 1))
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        so.sfc_moe_sort([0], t(9, dtype=I32), t(8, dtype=I32), t(8, dtype=I32))


@pytest.fixture
def as_if_on_the_gpu(monkeypatch):
    """Host tensors pass the device check, so that the checks behind it are reached."""
    monkeypatch.setattr(so, "_tensor", lambda t, name, what: None)

    def never(*a):
        raise AssertionError("reached the library")

    class Lib:
        def __getattr__(self, name):
            return never
    monkeypatch.setattr(so, "lib", Lib())


@pytest.mark.parametrize("error,match,f", [
    (TypeError, "float32 or bfloat16", lambda: so.sfc_mx4_quant(t(4, 32, dtype=torch.float16), u8(4, 16), u8(4, 1))),
    (ValueError, "2-D", lambda: so.sfc_mx4_quant(t(4), u8(4, 16), u8(4, 1))),
    (ValueError, "unit column stride", lambda: so.sfc_mx4_quant(t(32, 4).t(), u8(4, 16), u8(4, 1))),
    (ValueError, "no output", lambda: so.sfc_mx4_quant(t(4, 32))),
    (ValueError, "go together", lambda: so.sfc_mx4_quant(t(4, 32), u8(4, 16))),
    (ValueError, "shape mismatch", lambda: so.sfc_mx4_quant(t(4, 64), u8(4, 16), u8(4, 1))),
    (ValueError, "shape mismatch", lambda: so.sfc_mx4_quant(t(4, 32), u8(4, 16), u8(5, 1))),
    (ValueError, "shape mismatch", lambda: so.sfc_mx4_quant(t(4, 32), None, None, u8(4, 16), u8(4, 1))),
    (ValueError, "group of 4", lambda: so.sfc_mx4_quant(t(4, 32), u8(4, 16), u8(4, 1))),
    (ValueError, "topk", lambda: so.sfc_mx4_quant(t(4, 32), u8(4, 16), u8(4, 4)[:, :1], order=t(4, dtype=I32), topk=0)),
    (TypeError, "int32", lambda: so.sfc_mx4_quant(t(4, 32), u8(4, 16), u8(4, 4)[:, :1], order=t(4, dtype=torch.int64))),
    (TypeError, "uint8", lambda: so.sfc_mx4_dequant(t(4, 16), u8(4, 1), t(4, 32))),
    (ValueError, "shape mismatch", lambda: so.sfc_gemm_mx4_ex(*so.mx4_empty(4, 64, device="cpu"), *so.mx4_empty(8, 32, device="cpu"), t(4, 8))),
    (ValueError, "shape mismatch", lambda: so.sfc_gemm_mx4_ex(*so.mx4_empty(4, 64, device="cpu"), *so.mx4_empty(8, 64, device="cpu"), t(4, 9))),
    (ValueError, "shape mismatch", lambda: so.sfc_mx4_linear(t(4, 65), *so.mx4_empty(8, 64, device="cpu"), t(4, 8))),
    (ValueError, "elements", lambda: so.sfc_moe_sort(t(4, dtype=I32), t(9, dtype=I32), t(8, dtype=I32), t(5, dtype=I32))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(7, 32), topk=2)),
    (TypeError, "X's type", lambda: so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(8, 32, dtype=torch.float32), topk=2)),
    (ValueError, "elements", lambda: so.sfc_moe_dispatch(t(4, 32), t(8, dtype=I32), t(8, 32), topk=2, weights=t(7, dtype=torch.float32))),
    (ValueError, "multiple of 4 tokens", lambda: so.sfc_moe_combine(t(8, 32), t(7, dtype=I32), t(4, 32))),
    (TypeError, "weights must be float32", lambda: so.sfc_moe_combine(t(8, 32), t(8, dtype=I32), t(4, 32), weights=t(8))),
    (TypeError, "dY's type", lambda: so.sfc_moe_combine_grad(t(4, 32), t(8, 32, dtype=torch.float32), t(8, dtype=I32), t(8, dtype=I32), None,
                                                             t(8, 32), t(8, dtype=torch.float32))),
    (ValueError, "3-D", lambda: so.sfc_moe_gemm_mx4_ex(*so.mx4_empty(4, 64, device="cpu"), *so.mx4_empty(8, 64, device="cpu"), t(2, dtype=I32), t(4, 8))),
    (ValueError, "elements", lambda: so.sfc_moe_gemm_mx4_ex(*so.mx4_empty(4, 64, device="cpu"), *so.mx4_empty(8, 64, lead=(2,), device="cpu"),
                                                            t(2, dtype=I32), t(4, 8))),
    (ValueError, "3-D", lambda: so.sfc_moe_wgrad_mx4_ex(*so.mx4_empty(4, 64, device="cpu"), *so.mx4_empty(8, 64, device="cpu"), t(2, dtype=I32), t(4, 8))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_wgrad_mx4_ex(*so.mx4_empty(4, 64, device="cpu"), *so.mx4_empty(8, 64, device="cpu"),
                                                                   t(2, dtype=I32), t(2, 4, 8))),
])
def test_bad_operands_raise(as_if_on_the_gpu, error, match, f):
    with pytest.raises(error, match=match):
        f()
