"""Python binding of the 4-bit (MX) and mixture-of-experts operators of libsfcgemm.so.

Argument marshalling and checks only, as in ``sfcgemm``; names follow the C ABI
(include/sfcgemm.h, where each operator's definition stands).  Outputs are tensors
that the caller passes.

A 4-bit matrix of rows x cols values is a pair of uint8 tensors: codes (rows,
16 * ceil(cols/32)), two E2M1 codes to a byte, and scales (rows, ceil(cols/32)), E8M0;
rows of codes lie a multiple of 16 bytes apart, rows of scales a multiple of 4.
``mx4_empty`` allocates such a pair.

    xq = mx4_empty(M, K)
    sfc_mx4_quant(x, *xq)
    sfc_gemm_mx4_ex(*xq, *wq, y)            # y = x w^T
"""
from __future__ import annotations

import ctypes

import torch

from paper_2601_16294_amd.sfcgemm import SFC_OUT_BF16, SFC_OUT_F32, SFC_OK, SfcError, lib

try:
    from paper_2601_16294_amd import _sfcargs
except ImportError as e:
    raise ImportError("paper_2601_16294_amd/_sfcargs.so is not built; run `python -m paper_2601_16294_amd.build`") from e

__all__ = ["SfcError", "mx4_empty", "sfc_mx4_quant", "sfc_mx4_dequant", "sfc_gemm_mx4_ex", "sfc_mx4_linear",
           "sfc_gemm_mx4_ws_size", "sfc_mx4_linear_ws_size", "sfc_moe_sort", "sfc_moe_sort_rows", "sfc_moe_dispatch", "sfc_moe_combine", "sfc_moe_combine_grad",
           "sfc_moe_gemm_mx4_ex", "sfc_moe_wgrad_mx4_ex"]


def _declare() -> None:
    i64, i32, p, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    mx = [p, i64, p, i64]                        # codes, row bytes, scales, row bytes
    rows = [p, i64]                              # matrix, leading dimension
    lib.sfc_mx4_quant.argtypes = [i64, i64] + rows + [i32, p, i64, i32] + mx + mx + [p]
    lib.sfc_mx4_dequant.argtypes = [i64, i64] + mx + rows + [i32, p]
    lib.sfc_gemm_mx4_ex.argtypes = [i64, i64, i64] + mx + mx + rows + [i32, p]
    lib.sfc_mx4_linear.argtypes = [i64, i64, i64] + rows + [i32] + mx + rows + [i32, p]
    lib.sfc_gemm_mx4_ws_ex.argtypes = lib.sfc_gemm_mx4_ex.argtypes[:-1] + [p, sz, p]
    lib.sfc_mx4_linear_ws.argtypes = lib.sfc_mx4_linear.argtypes[:-1] + [p, sz, p]
    lib.sfc_gemm_mx4_ws_size.argtypes = lib.sfc_mx4_linear_ws_size.argtypes = [i64, i64, i64, i32]
    lib.sfc_moe_sort_ws_size.argtypes = [i64, i32]
    lib.sfc_moe_sort.argtypes = [i64, i32, i32, p, i64, p, p, p, p, sz, p]
    lib.sfc_moe_dispatch.argtypes = [i64, i64, i64, i32] + rows + [i32, p, p] + rows + [p]
    lib.sfc_moe_combine.argtypes = [i64, i64, i64, i32] + rows + [i32, p, p] + rows + [p]
    lib.sfc_moe_combine_grad.argtypes = [i64, i64, i64, i32] + rows + rows + [i32, p, p, p] + rows + [p, p]
    lib.sfc_moe_gemm_mx4_ex.argtypes = [i64, i64, i64, i32] + mx + [p, i64, i64, p, i64, i64, p] + rows + [i32, p]
    lib.sfc_moe_wgrad_mx4_ex.argtypes = [i64, i64, i64, i32] + mx + mx + [p] + rows + [i64, i32, p]
    for name in __all__:
        if name.startswith("sfc_") and name != "sfc_moe_sort_rows" and not name.endswith("_size"):
            getattr(lib, name).restype = i32
    for name in ("sfc_gemm_mx4_ws_ex", "sfc_mx4_linear_ws"):
        getattr(lib, name).restype = i32
    for name in ("sfc_gemm_mx4_ws_size", "sfc_mx4_linear_ws_size", "sfc_moe_sort_ws_size"):
        getattr(lib, name).restype = sz


_declare()


_TYPES = {torch.float32: SFC_OUT_F32, torch.bfloat16: SFC_OUT_BF16}
_Tensor, _U8, _I32, _F32 = torch.Tensor, torch.uint8, torch.int32, torch.float32
# (the accessors behind torch.cuda.current_device and current_stream; a small call is bound by
# its host time)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


# Each gives what the function of its name below gives where the argument is as it should be, else
# None: the code behind it then names the fault.
_rows_of, _mx4_of, _vector_of, _empty_of = _sfcargs.rows, _sfcargs.mx4, _sfcargs.vector, _sfcargs.empty
_ANY = (-1, -1)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_current()) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _check(code: int, what: str) -> None:
    if code != SFC_OK:
        raise SfcError(code, what)


def _tensor(t, name, what):
    if not isinstance(t, _Tensor):
        raise TypeError(f"{what}: {name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{what}: {name} must be a CUDA tensor (got {t.device})")
    if t.get_device() != _current():
        raise ValueError(f"{what}: {name} is on {t.device}, the current device is cuda:{_current()}")


def _rows(t, name, what, shape=None):
    """(pointer, leading dimension, type code) of a 2-D fp32 or bf16 tensor with unit column stride."""
    got = _rows_of(t, *(shape or _ANY))
    if got is not None:
        return got
    _tensor(t, name, what)
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: {name} must be float32 or bfloat16 (got {t.dtype})")
    s = t.stride()
    if len(s) != 2:
        raise ValueError(f"{what}: {name} must be 2-D")
    r, c = t.shape
    if shape is not None and (r != shape[0] or c != shape[1]):
        raise ValueError(f"{what}: shape mismatch: {name} is {tuple(t.shape)}, expected {tuple(shape)}")
    if s[1] != 1 and c > 1:
        raise ValueError(f"{what}: {name} must have unit column stride")
    return t.data_ptr(), s[0] if r > 1 else c or 1, code


def _mx4(q, s, name, what, rows=None, cols=None, lead=0):
    """(codes, row bytes, scales, row bytes) of a 4-bit matrix, `lead` dimensions before it.
    Checks the shape against rows x cols where they are given."""
    if cols is None:
        got = _mx4_of(q, s, lead, -1, -1)
    else:
        got = _mx4_of(q, s, lead, -1 if rows is None else rows, (cols + 31) // 32)
    if got is not None:
        return got
    _tensor(q, name, what)
    _tensor(s, f"{name}'s scales", what)
    if q.dtype != _U8 or s.dtype != _U8:
        raise TypeError(f"{what}: {name} and its scales must be uint8 (got {q.dtype} and {s.dtype})")
    sq, ss, dq, ds = q.shape, s.shape, q.stride(), s.stride()
    if len(sq) != 2 + lead or len(ss) != 2 + lead:
        raise ValueError(f"{what}: {name} and its scales must be {2 + lead}-D")
    r, half, blocks = sq[-2], sq[-1], ss[-1]
    if half != 16 * blocks or ss[-2] != r or (lead and ss[0] != sq[0]):
        raise ValueError(f"{what}: shape mismatch: {name} {tuple(sq)} and its scales {tuple(ss)} "
                         "(16 bytes of codes to a scale)")
    if (dq[-1] != 1 and half > 1) or (ds[-1] != 1 and blocks > 1):
        raise ValueError(f"{what}: {name} and its scales must have unit column stride")
    if cols is not None and ((rows is not None and r != rows) or blocks != (cols + 31) // 32):
        raise ValueError(f"{what}: shape mismatch: {name} is {tuple(sq)}, expected "
                         f"{(r if rows is None else rows, 16 * ((cols + 31) // 32))}")
    padded = (blocks + 3) & ~3
    if padded != blocks and q.numel():
        # the last row of scales, too, is read in whole groups of 4
        last = s.storage_offset() + sum((n - 1) * d for n, d in zip(ss[:-1], ds[:-1]))
        if last + padded > s.untyped_storage().nbytes():
            raise ValueError(f"{what}: the scales of {name} end inside a group of 4 bytes: allocate rows of "
                             f"{padded} (mx4_empty does)")
    if r > 1:
        return q.data_ptr(), dq[-2], s.data_ptr(), ds[-2]
    return q.data_ptr(), half or 16, s.data_ptr(), padded or 4


def _vector(t, name, what, dtype, count):
    """Pointer of a contiguous tensor of `count` elements (None: any number)."""
    got = _vector_of(t, dtype is _F32, -1 if count is None else count)
    if got is not None:
        return got
    _tensor(t, name, what)
    if t.dtype != dtype:
        raise TypeError(f"{what}: {name} must be {str(dtype)[6:]} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{what}: {name} must be contiguous")
    if count is not None and t.numel() != count:
        raise ValueError(f"{what}: {name} has {t.numel()} elements, expected {count}")
    return t.data_ptr()


def _ints(t, name, what, count):
    return _vector(t, name, what, _I32, count)


def _weights(t, what, count):
    return None if t is None else _vector(t, "weights", what, _F32, count)


def _memory(t, what):
    """(pointer, bytes) of a caller's workspace, a contiguous tensor of any type.  An empty one, which has
    no pointer, is still the caller's: no call that needs memory takes it."""
    _tensor(t, "workspace", what)
    if not t.is_contiguous():
        raise ValueError(f"{what}: workspace must be contiguous")
    return t.data_ptr() or 16, t.numel() * t.element_size()


def _int(v, name, what):
    """v, if it fits a C int (ctypes would cut it to 32 bits)."""
    if not -(1 << 31) <= v < 1 << 31:
        raise ValueError(f"{what}: {name} must be < 2^31 (got {v})")
    return v


def _topk(topk, what):
    if topk < 1:
        raise ValueError(f"{what}: topk must be >= 1")
    return _int(topk, "topk", what)


def mx4_empty(rows: int, cols: int, lead=(), device="cuda"):
    """Uninitialised (codes, scales) of a rows x cols 4-bit matrix (or of `lead` such matrices)."""
    if lead == () and device == "cuda":
        got = _empty_of(rows, cols)
        if got is not None:
            return got
    b = (cols + 31) // 32
    padded = (b + 3) & ~3
    codes = torch.empty((*lead, rows, 16 * b), dtype=_U8, device=device)
    scales = torch.empty((*lead, rows, padded), dtype=_U8, device=device)
    return codes, scales if padded == b else scales[..., :b]


def sfc_mx4_quant(X, Q=None, S=None, Qt=None, St=None, order=None, topk: int = 1, stream=None) -> None:
    """X (rows, cols) to 4 bits: Q, S with blocks along the rows, and / or Qt, St (cols, rows),
    transposed with blocks along the columns.  With `order` (sfc_moe_sort's) the rows are
    X[order // topk], zeros where order is negative."""
    what = "sfc_mx4_quant"
    px, ldx, kind = _rows(X, "X", what)
    x_rows, cols = X.shape
    rows, po = x_rows, None
    if order is not None:
        po, rows = _ints(order, "order", what, None), order.numel()
        _topk(topk, what)
    if (Q is None) != (S is None) or (Qt is None) != (St is None):
        raise ValueError(f"{what}: codes and scales go together")
    if Q is None and Qt is None:
        raise ValueError(f"{what}: no output")
    a = _mx4(Q, S, "Q", what, rows, cols) if Q is not None else (None, 0, None, 0)
    b = _mx4(Qt, St, "Qt", what, cols, rows) if Qt is not None else (None, 0, None, 0)
    _check(lib.sfc_mx4_quant(rows, cols, px, ldx, kind, po, x_rows, topk, *a, *b, _stream(stream)), what)


def sfc_mx4_dequant(Q, S, Y, stream=None) -> None:
    """Y (rows, cols), float32 or bfloat16, = the values of the 4-bit matrix (Q, S)."""
    what = "sfc_mx4_dequant"
    py, ldy, kind = _rows(Y, "Y", what)
    rows, cols = Y.shape
    _check(lib.sfc_mx4_dequant(rows, cols, *_mx4(Q, S, "Q", what, rows, cols), py, ldy, kind, _stream(stream)),
           what)


def sfc_gemm_mx4_ws_size(M: int, N: int, K: int, dtype=torch.float32) -> int:
    """Bytes of the workspace that sfc_gemm_mx4_ex takes for an output of `dtype` (0: none)."""
    return int(lib.sfc_gemm_mx4_ws_size(M, N, K, _TYPES[dtype]))


def sfc_mx4_linear_ws_size(M: int, N: int, K: int, dtype=torch.float32) -> int:
    """As sfc_gemm_mx4_ws_size, for sfc_mx4_linear."""
    return int(lib.sfc_mx4_linear_ws_size(M, N, K, _TYPES[dtype]))


def sfc_gemm_mx4_ex(A, As, B, Bs, C, stream=None, workspace=None) -> None:
    """C (M, N), float32 or bfloat16, = A B^T with A (M, K) and B (N, K) in 4 bits.  workspace: None
    (library memory of the stream) or a tensor of sfc_gemm_mx4_ws_size() bytes."""
    what = "sfc_gemm_mx4_ex"
    a, b = _mx4(A, As, "A", what), _mx4(B, Bs, "B", what)
    M, K, N = A.shape[0], 32 * As.shape[1], B.shape[0]
    if Bs.shape[1] != As.shape[1]:
        raise ValueError(f"{what}: shape mismatch: A {tuple(A.shape)} B {tuple(B.shape)}")
    pc, ldc, kind = _rows(C, "C", what, (M, N))
    if workspace is not None:
        return _check(lib.sfc_gemm_mx4_ws_ex(M, N, K, *a, *b, pc, ldc, kind, *_memory(workspace, what), _stream(stream)), what)
    _check(lib.sfc_gemm_mx4_ex(M, N, K, *a, *b, pc, ldc, kind, _stream(stream)), what)


def sfc_mx4_linear(X, W, Ws, Y, stream=None, workspace=None) -> None:
    """Y (M, N) = X W^T with X (M, K), float32 or bfloat16, brought to 4 bits in the call and
    W (N, K) in 4 bits.  workspace: None or a tensor of sfc_mx4_linear_ws_size() bytes; graphs
    that are replayed at once need workspaces of their own."""
    what = "sfc_mx4_linear"
    px, ldx, kind = _rows(X, "X", what)
    M, K = X.shape
    w = _mx4(W, Ws, "W", what, cols=K)
    N = W.shape[0]
    py, ldy, out = _rows(Y, "Y", what, (M, N))
    if workspace is not None:
        return _check(lib.sfc_mx4_linear_ws(M, N, K, px, ldx, kind, *w, py, ldy, out, *_memory(workspace, what), _stream(stream)),
                      what)
    _check(lib.sfc_mx4_linear(M, N, K, px, ldx, kind, *w, py, ldy, out, _stream(stream)), what)


def sfc_moe_sort_rows(slots: int, experts: int, align: int = 1) -> int:
    """Rows that sorted arrays need: every slot, and the padding of each expert's rows."""
    return slots + experts * (align - 1)


def sfc_moe_sort(ids, offsets, order, pos, align: int = 1, workspace=None, stream=None) -> None:
    """Slots sorted by expert.  ids (int32, any shape; slot = flat index), offsets
    (experts + 1,), order (at least sfc_moe_sort_rows(...),), pos (as many as ids): int32."""
    what = "sfc_moe_sort"
    pi, slots = _ints(ids, "ids", what, None), ids.numel()
    pp = _ints(pos, "pos", what, slots)
    po, pr = _ints(offsets, "offsets", what, None), _ints(order, "order", what, None)
    ws, ws_bytes = None, 0
    if workspace is not None:
        ws, ws_bytes = _memory(workspace, what)
    experts = _int(offsets.numel() - 1, "the number of experts", what)
    _check(lib.sfc_moe_sort(slots, experts, _int(align, "align", what), pi, order.numel(), po, pr, pp, ws, ws_bytes,
                            _stream(stream)), what)


def sfc_moe_dispatch(X, order, Xs, topk: int = 1, weights=None, stream=None) -> None:
    """Xs (rows, cols) = the tokens' rows in sorted order, X (tokens, cols); times weights
    (float32, tokens * topk) if given."""
    what = "sfc_moe_dispatch"
    px, ldx, kind = _rows(X, "X", what)
    tokens, cols = X.shape
    po, rows = _ints(order, "order", what, None), order.numel()
    ps, lds, out = _rows(Xs, "Xs", what, (rows, cols))
    if out != kind:
        raise TypeError(f"{what}: Xs must hold X's type")
    _check(lib.sfc_moe_dispatch(rows, cols, tokens, _topk(topk, what), px, ldx, kind, po,
                                _weights(weights, what, tokens * topk), ps, lds, _stream(stream)), what)


def sfc_moe_combine(Ys, pos, Y, weights=None, stream=None) -> None:
    """Y (tokens, cols) = sum over a token's slots of weights * Ys[pos]; Ys (rows, cols), pos
    and weights of tokens * topk elements, the topk slots of a token side by side."""
    what = "sfc_moe_combine"
    pr, ldr, kind = _rows(Ys, "Ys", what)
    rows, cols = Ys.shape
    py, ldy, out = _rows(Y, "Y", what)
    tokens = Y.shape[0]
    if Y.shape[1] != cols:
        raise ValueError(f"{what}: shape mismatch: Ys {tuple(Ys.shape)} Y {tuple(Y.shape)}")
    if out != kind:
        raise TypeError(f"{what}: Y must hold Ys's type")
    pp, slots = _ints(pos, "pos", what, None), pos.numel()
    topk = _slots_per_token(slots, tokens, what)
    _check(lib.sfc_moe_combine(tokens, cols, rows, topk, pr, ldr, kind, pp,
                               _weights(weights, what, slots), py, ldy, _stream(stream)), what)


def _slots_per_token(slots, tokens, what):
    if tokens == 0:
        if slots:
            raise ValueError(f"{what}: pos has {slots} elements, expected 0")
        return 1
    if slots == 0 or slots % tokens:
        raise ValueError(f"{what}: pos has {slots} elements, expected a multiple of {tokens} tokens")
    return _int(slots // tokens, "topk", what)


def sfc_moe_combine_grad(dY, Ys, order, pos, weights, dYs, dW, stream=None) -> None:
    """Gradient of sfc_moe_combine: dYs (rows, cols) and dW (float32, tokens * topk) from dY
    (tokens, cols), Ys (rows, cols) and weights (or None: 1)."""
    what = "sfc_moe_combine_grad"
    pd, ldd, kind = _rows(dY, "dY", what)
    tokens, cols = dY.shape
    pr, ldr, kr = _rows(Ys, "Ys", what)
    rows = Ys.shape[0]
    if Ys.shape[1] != cols:
        raise ValueError(f"{what}: shape mismatch: dY {tuple(dY.shape)} Ys {tuple(Ys.shape)}")
    ps, lds, ks = _rows(dYs, "dYs", what, (rows, cols))
    if kr != kind or ks != kind:
        raise TypeError(f"{what}: Ys and dYs must hold dY's type")
    pp, slots = _ints(pos, "pos", what, None), pos.numel()
    topk = _slots_per_token(slots, tokens, what)
    _check(lib.sfc_moe_combine_grad(tokens, cols, rows, topk, pd, ldd, pr, ldr, kind, _ints(order, "order", what, rows),
                                    pp, _weights(weights, what, slots), ps, lds,
                                    _vector(dW, "dW", what, _F32, slots), _stream(stream)), what)


def sfc_moe_gemm_mx4_ex(A, As, B, Bs, offsets, C, stream=None) -> None:
    """C (rows, N) = A (rows, K) times, row by row, the transposed B (experts, N, K) of the row's
    expert; rows offsets[e] .. offsets[e+1]-1 are expert e's.  4-bit operands."""
    what = "sfc_moe_gemm_mx4_ex"
    a, b = _mx4(A, As, "A", what), _mx4(B, Bs, "B", what, lead=1)
    rows, K, E, N = A.shape[0], 32 * As.shape[1], _int(B.shape[0], "the number of experts", what), B.shape[1]
    if Bs.shape[2] != As.shape[1]:
        raise ValueError(f"{what}: shape mismatch: A {tuple(A.shape)} B {tuple(B.shape)}")
    pc, ldc, kind = _rows(C, "C", what, (rows, N))
    _check(lib.sfc_moe_gemm_mx4_ex(rows, N, K, E, *a, b[0], b[1], B.stride(0), b[2], b[3], Bs.stride(0),
                                   _ints(offsets, "offsets", what, E + 1), pc, ldc, kind, _stream(stream)), what)


def sfc_moe_wgrad_mx4_ex(A, As, B, Bs, offsets, C, stream=None) -> None:
    """C (experts, M, N), C[e] = A[:, seg] B[:, seg]^T over the sorted rows seg of expert e (starts
    multiples of 32); A (M, rows) and B (N, rows) in 4 bits, blocks along the rows."""
    what = "sfc_moe_wgrad_mx4_ex"
    a, b = _mx4(A, As, "A", what), _mx4(B, Bs, "B", what)
    M, N, rows = A.shape[0], B.shape[0], 32 * As.shape[1]
    if Bs.shape[1] != As.shape[1]:
        raise ValueError(f"{what}: shape mismatch: A {tuple(A.shape)} B {tuple(B.shape)}")
    if not isinstance(C, _Tensor) or C.dim() != 3:
        raise ValueError(f"{what}: C must be a 3-D tensor")
    E = _int(C.shape[0], "the number of experts", what)
    po = _ints(offsets, "offsets", what, None)
    if E < 1 or offsets.numel() != E + 1 or C.shape[1] != M or C.shape[2] != N:
        raise ValueError(f"{what}: shape mismatch: A {tuple(A.shape)} B {tuple(B.shape)} offsets "
                         f"{tuple(offsets.shape)} C {tuple(C.shape)}")
    pc, ldc, kind = _rows(C[0], "C", what, (M, N))
    _check(lib.sfc_moe_wgrad_mx4_ex(M, N, rows, E, *a, *b, po, pc, ldc, C.stride(0), kind, _stream(stream)), what)
