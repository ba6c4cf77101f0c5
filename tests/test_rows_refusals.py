"""The experts' bf16 products and the low-rank adapters refuse bad arguments before any HIP call: wrong sizes,
strides, alignment, types and devices, at the C ABI and at the Python binding.  No GPU is needed."""
import pytest
import torch

from paper_2601_16294_amd import sfcops as so

lib = so.lib
F32, BF16 = 0, 1
NK, KN = so.SFC_B_NK, so.SFC_B_KN
A, B, C, O, S, V = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000


def call(fn, order, good, kw):
    a = dict(good)
    a.update(kw)
    return fn(*[a[k] for k in order.split()])


GEMM = "rows N K experts A lda order a_rows topk B ldb stride layout offsets C ldc type stream"
GGOOD = dict(rows=8, N=12, K=20, experts=3, A=A, lda=20, order=None, a_rows=0, topk=0, B=B, ldb=20, stride=240, layout=NK, offsets=O,
             C=C, ldc=12, type=F32, stream=None)
WGRAD = "M N rows experts A lda B ldb offsets C ldc stride type stream"
WGOOD = dict(M=12, N=20, rows=8, experts=3, A=A, lda=12, B=B, ldb=20, offsets=O, C=C, ldc=20, stride=240, type=F32, stream=None)
DOWN = "rows K rank adapters X ldx A lda stride layout ids scales V ldv ws bytes stream"
DGOOD = dict(rows=8, K=20, rank=4, adapters=3, X=A, ldx=20, A=B, lda=20, stride=80, layout=NK, ids=O, scales=S, V=V, ldv=4, ws=None,
             bytes=0, stream=None)
UP = "rows N rank adapters V ldv B ldb stride layout ids base ldbase Y ldy type stream"
UGOOD = dict(rows=8, N=20, rank=4, adapters=3, V=V, ldv=4, B=B, ldb=4, stride=80, layout=NK, ids=O, base=A, ldbase=20, Y=C, ldy=20,
             type=F32, stream=None)
GRAD = "rows columns rank adapters Z ldz V ldv ids G ldg stride layout type ws bytes stream"
RGOOD = dict(rows=8, columns=20, rank=4, adapters=3, Z=A, ldz=20, V=V, ldv=4, ids=O, G=C, ldg=4, stride=80, layout=NK, type=F32,
             ws=None, bytes=0, stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(N=-1), -1), (dict(K=-1), -1), (dict(rows=1 << 31), -2), (dict(N=1 << 31), -2), (dict(K=1 << 31), -2),
    (dict(experts=0), -1), (dict(experts=-1), -1), (dict(experts=1025), -2), (dict(layout=2), -1), (dict(layout=-1), -1),
    (dict(type=2), -1), (dict(A=None), -1), (dict(B=None), -1), (dict(C=None), -1), (dict(offsets=None), -1), (dict(lda=19), -1),
    (dict(ldb=19), -1), (dict(ldc=11), -1), (dict(layout=KN, ldb=11), -1), (dict(stride=-1), -1), (dict(A=A + 1), -2), (dict(B=B + 1), -2),
    (dict(C=C + 2), -2), (dict(type=BF16, C=C + 1), -2), (dict(offsets=O + 2), -2), (dict(lda=1 << 22), -2), (dict(ldb=1 << 22), -2),
    (dict(order=O, a_rows=4, topk=0), -1), (dict(order=O, a_rows=4, topk=-2), -1), (dict(order=O, a_rows=-1, topk=1), -1),
    (dict(order=O + 1, a_rows=4, topk=1), -2), (dict(order=O, a_rows=1 << 31, topk=1), -2),
    (dict(order=O, a_rows=1 << 20, lda=1 << 11, topk=1), -2), (dict(order=O, a_rows=0, topk=0), -1),
    (dict(rows=(1 << 31) - 1, N=(1 << 31) - 1, ldc=(1 << 31) - 1), -2)])
def test_experts(kw, code):
    assert call(lib.sfc_moe_gemm_ex, GEMM, GGOOD, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(M=-1), -1), (dict(N=-1), -1), (dict(M=1 << 31), -2), (dict(experts=0), -1), (dict(experts=1025), -2),
    (dict(type=3), -1), (dict(A=None), -1), (dict(B=None), -1), (dict(C=None), -1), (dict(offsets=None), -1), (dict(lda=11), -1),
    (dict(ldb=19), -1), (dict(ldc=19), -1), (dict(A=A + 1), -2), (dict(B=B + 1), -2), (dict(C=C + 2), -2), (dict(offsets=O + 1), -2),
    (dict(lda=1 << 22), -2), (dict(ldb=1 << 22), -2), (dict(stride=239), -1), (dict(stride=0), -1), (dict(stride=-240), -1),
    (dict(stride=20, ldc=59), -1), (dict(stride=19, ldc=60), -1), (dict(stride=1 << 62, ldc=1 << 62), -1),
    (dict(M=1 << 21, N=1 << 21, lda=1 << 21, ldb=1 << 21, ldc=1 << 21, stride=1 << 42, experts=1024), -2)])
def test_experts_weight_gradient(kw, code):
    assert call(lib.sfc_moe_wgrad_ex, WGRAD, WGOOD, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(K=-1), -1), (dict(rank=-1), -1), (dict(rank=257, lda=300, ldv=300), -2), (dict(adapters=0), -1),
    (dict(adapters=-5), -1), (dict(layout=2), -1), (dict(rows=1 << 31), -2), (dict(X=None), -1), (dict(A=None), -1), (dict(V=None), -1),
    (dict(ids=None), -1), (dict(ldx=19), -1), (dict(lda=19), -1), (dict(layout=KN, lda=3), -1), (dict(ldv=3), -1), (dict(stride=-1), -1),
    (dict(X=A + 1), -2), (dict(A=B + 1), -2), (dict(V=V + 2), -2), (dict(ids=O + 2), -2), (dict(scales=S + 2), -2),
    (dict(ldx=1 << 22), -2), (dict(lda=1 << 22), -2), (dict(ws=V + 8, bytes=1 << 30), -2)])
def test_down(kw, code):
    assert call(lib.sfc_lora_down, DOWN, DGOOD, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(N=-1), -1), (dict(rank=-1), -1), (dict(rank=257, ldb=300, ldv=300), -2), (dict(adapters=0), -1),
    (dict(layout=7), -1), (dict(type=2), -1), (dict(rows=1 << 31), -2), (dict(V=None), -1), (dict(B=None), -1), (dict(Y=None), -1),
    (dict(ids=None), -1), (dict(ldv=3), -1), (dict(ldb=3), -1), (dict(layout=KN, ldb=19), -1), (dict(ldy=19), -1), (dict(ldbase=19), -1),
    (dict(stride=-1), -1), (dict(V=V + 2), -2), (dict(B=B + 1), -2), (dict(Y=C + 2), -2), (dict(type=BF16, Y=C + 1), -2),
    (dict(base=A + 2), -2), (dict(type=BF16, base=A + 1), -2), (dict(ids=O + 2), -2), (dict(base=C, ldbase=24), -1)])
def test_up(kw, code):
    assert call(lib.sfc_lora_up, UP, UGOOD, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(columns=-1), -1), (dict(rank=-1), -1), (dict(rank=257, ldg=300, ldv=300, stride=1 << 20), -2),
    (dict(adapters=0), -1), (dict(layout=7), -1), (dict(type=2), -1), (dict(rows=1 << 31), -2), (dict(Z=None), -1), (dict(V=None), -1),
    (dict(G=None), -1), (dict(ids=None), -1), (dict(ldz=19), -1), (dict(ldv=3), -1), (dict(ldg=3), -1), (dict(layout=KN, ldg=19), -1),
    (dict(stride=79), -1), (dict(stride=0), -1), (dict(stride=4, ldg=11), -1), (dict(Z=A + 1), -2), (dict(V=V + 2), -2),
    (dict(G=C + 2), -2), (dict(type=BF16, G=C + 1), -2), (dict(ids=O + 2), -2), (dict(ws=V + 8, bytes=1 << 30), -2)])
def test_adapters_weight_gradient(kw, code):
    assert call(lib.sfc_lora_wgrad, GRAD, RGOOD, kw) == code


def test_nothing_to_do_is_success():
    assert call(lib.sfc_moe_gemm_ex, GEMM, GGOOD, dict(rows=0, A=None, C=None)) == 0
    assert call(lib.sfc_moe_gemm_ex, GEMM, GGOOD, dict(N=0, B=None, C=None)) == 0
    assert call(lib.sfc_moe_wgrad_ex, WGRAD, WGOOD, dict(M=0, A=None, C=None)) == 0
    assert call(lib.sfc_lora_down, DOWN, DGOOD, dict(rows=0, X=None, V=None, ids=None)) == 0
    assert call(lib.sfc_lora_down, DOWN, DGOOD, dict(rank=0, A=None, V=None)) == 0
    assert call(lib.sfc_lora_up, UP, UGOOD, dict(rows=0, V=None, Y=None, ids=None)) == 0
    assert call(lib.sfc_lora_up, UP, UGOOD, dict(N=0, B=None, Y=None, base=None)) == 0
    assert call(lib.sfc_lora_wgrad, GRAD, RGOOD, dict(columns=0, Z=None, G=None)) == 0
    assert call(lib.sfc_lora_wgrad, GRAD, RGOOD, dict(rank=0, V=None, G=None)) == 0


@pytest.mark.parametrize("f", [lib.sfc_lora_down_ws_size, lib.sfc_lora_wgrad_ws_size])
@pytest.mark.parametrize("sizes", [(-1, 64, 16, 2), (64, -1, 16, 2), (64, 64, -1, 2), (64, 64, 257, 2), (64, 64, 16, 0), (1 << 31, 64, 16, 2),
                                   (64, 64, 0, 2)])
def test_bad_sizes_need_no_workspace(f, sizes):
    assert f(*sizes) == 0


# ---- the binding: host tensors, wrong types and shapes never reach the library -------------------


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


I32, FP = torch.int32, torch.float32


def ints(n):
    return t(n, dtype=I32)


@pytest.mark.parametrize("f", [
    lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8)),
    lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8), ints(3), t(2, 16, 8, dtype=FP)),
    lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(4), t(4, 8, dtype=FP)),
    lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 32, 8), ints(4), t(4, 32)),
    lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8, dtype=FP), ints(4), t(2, 32, 8)),
])
def test_host_tensors_raise(f):
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        f()


def test_non_tensors_raise():
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        so.sfc_moe_gemm_ex([1.0], t(2, 8, 32), ints(3), t(4, 8))
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        so.sfc_lora_wgrad(None, t(4, 8, dtype=FP), ints(4), t(2, 32, 8))


@pytest.fixture
def calls(monkeypatch):
    """Host tensors pass the device check, so that the checks behind it are reached; what reaches the library is kept."""
    got = []
    monkeypatch.setattr(so, "_tensor", lambda t, name, what: None)
    monkeypatch.setattr(so, "_stream", lambda s: None)

    class Lib:
        def __getattr__(self, name):
            return lambda *a: got.append((name, a)) or 0
    monkeypatch.setattr(so, "lib", Lib())
    return got


@pytest.mark.parametrize("error,match,f", [
    (TypeError, "bfloat16", lambda: so.sfc_moe_gemm_ex(t(4, 32, dtype=FP), t(2, 8, 32), ints(3), t(4, 8))),
    (TypeError, "float32 or bfloat16", lambda: so.sfc_moe_gemm_ex(t(4, 32, dtype=torch.float16), t(2, 8, 32), ints(3), t(4, 8))),
    (TypeError, "bfloat16", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32, dtype=FP), ints(3), t(4, 8))),
    (TypeError, "float32 or bfloat16", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8, dtype=torch.float16))),
    (TypeError, "int32", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), t(3, dtype=torch.int64), t(4, 8))),
    (ValueError, "elements", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(2), t(4, 8))),
    (ValueError, "3-D", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(8, 32), ints(3), t(4, 8))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 32, 8), ints(3), t(4, 8))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8), layout=KN)),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 9))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8), order=ints(5))),
    (ValueError, "layout", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8), layout=2)),
    (ValueError, "unit column stride", lambda: so.sfc_moe_gemm_ex(t(32, 4).t(), t(2, 8, 32), ints(3), t(4, 8))),
    (ValueError, "unit column stride", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 32, 8).transpose(1, 2), ints(3), t(4, 8))),
    (ValueError, "topk", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8), order=ints(4), topk=0)),
    (TypeError, "int32", lambda: so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8), order=t(4, dtype=torch.int64))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(5, 8), ints(3), t(2, 16, 8))),
    (ValueError, "shape mismatch", lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8), ints(3), t(2, 8, 16))),
    (ValueError, "3-D", lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8), ints(2), t(16, 8))),
    (ValueError, "elements", lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8), ints(2), t(2, 16, 8))),
    (TypeError, "bfloat16", lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8, dtype=FP), ints(3), t(2, 16, 8))),
    (TypeError, "float32 or bfloat16", lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8), ints(3), t(2, 16, 8, dtype=torch.float16))),
    (TypeError, "float32", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(4), t(4, 8))),
    (TypeError, "bfloat16", lambda: so.sfc_lora_down(t(4, 32, dtype=FP), t(2, 8, 32), ints(4), t(4, 8, dtype=FP))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 33), ints(4), t(4, 8, dtype=FP))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(4), t(4, 9, dtype=FP))),
    (ValueError, "elements", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(5), t(4, 8, dtype=FP))),
    (TypeError, "int32", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), t(4, dtype=torch.int64), t(4, 8, dtype=FP))),
    (ValueError, "elements", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(4), t(4, 8, dtype=FP), scales=t(3, dtype=FP))),
    (TypeError, "float32", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(4), t(4, 8, dtype=FP), scales=t(2))),
    (ValueError, "layout", lambda: so.sfc_lora_down(t(4, 32), t(2, 8, 32), ints(4), t(4, 8, dtype=FP), layout=None)),
    (TypeError, "float32", lambda: so.sfc_lora_up(t(4, 8), t(2, 32, 8), ints(4), t(4, 32))),
    (TypeError, "bfloat16", lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 32, 8, dtype=FP), ints(4), t(4, 32))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 8, 32), ints(4), t(4, 32))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 32, 8), ints(4), t(4, 33))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 32, 8), ints(4), t(4, 32), base=t(5, 32))),
    (TypeError, "Y's type", lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 32, 8), ints(4), t(4, 32), base=t(4, 32, dtype=FP))),
    (ValueError, "elements", lambda: so.sfc_lora_up(t(4, 8, dtype=FP), t(2, 32, 8), ints(3), t(4, 32))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_wgrad(t(4, 32), t(5, 8, dtype=FP), ints(4), t(2, 32, 8))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8, dtype=FP), ints(4), t(2, 8, 32))),
    (ValueError, "shape mismatch", lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8, dtype=FP), ints(4), t(2, 32, 8), layout=KN)),
    (ValueError, "layout", lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8, dtype=FP), ints(4), t(2, 32, 8), layout=5)),
    (TypeError, "float32", lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8), ints(4), t(2, 32, 8))),
    (ValueError, "elements", lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8, dtype=FP), ints(5), t(2, 32, 8))),
])
def test_bad_operands_raise(calls, error, match, f):
    with pytest.raises(error, match=match):
        f()
    assert calls == []


def test_counts_past_32_bits_raise(calls, monkeypatch):
    """Counts that come from a tensor's shape: cut to 32 bits, 2^32 + 2 matrices would pass for 2."""
    n = (1 << 32) + 2
    monkeypatch.setattr(so, "_ints", lambda t, name, what, count: 0)
    many = lambda r, c: t(1, r, c).expand(n, r, c)
    for f in (lambda: so.sfc_moe_gemm_ex(t(4, 32), many(8, 32), ints(3), t(4, 8)),
              lambda: so.sfc_moe_wgrad_ex(t(4, 16), t(4, 8), ints(3), many(16, 8)),
              lambda: so.sfc_lora_down(t(4, 32), many(8, 32), ints(4), t(4, 8, dtype=FP)),
              lambda: so.sfc_lora_up(t(4, 8, dtype=FP), many(32, 8), ints(4), t(4, 32)),
              lambda: so.sfc_lora_wgrad(t(4, 32), t(4, 8, dtype=FP), ints(4), many(32, 8))):
        with pytest.raises(ValueError, match=r"2\^31"):
            f()
    assert calls == []
    with pytest.raises(ValueError, match=r"2\^31"):
        so.sfc_moe_gemm_ex(t(4, 32), t(2, 8, 32), ints(3), t(4, 8), order=ints(4), topk=n)
