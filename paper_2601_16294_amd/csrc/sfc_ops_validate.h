// Argument checks of the 4-bit and expert entry points, free of any HIP dependency; every
// check happens before the library touches the device.
#pragma once
#include <stdint.h>

#include "sfc_validate.h"

namespace sfc {

constexpr int64_t kMxMaxStride = (int64_t)1 << 22;    // bytes: 256 rows stay within 32-bit offsets

inline bool type_ok(int type) { return type == SFC_OUT_F32 || type == SFC_OUT_BF16; }
inline int64_t type_size(int type) { return type == SFC_OUT_F32 ? 4 : 2; }
inline int64_t mx4_blocks(int64_t cols) { return cols / 32 + (cols % 32 != 0); }

// A matrix of fp32 or bf16 elements.
inline Checked check_rows(const void* p, int64_t rows, int64_t cols, int64_t ld, int type, const char* null_text,
                          const char* ld_text) {
  if (rows == 0 || cols == 0) return ok();
  if (!p) return fail(SFC_ERR_INVALID_ARG, null_text);
  if (ld < cols) return fail(SFC_ERR_INVALID_ARG, ld_text);
  if ((uintptr_t)p % type_size(type)) return fail(SFC_ERR_UNSUPPORTED, "a matrix is not aligned to its element size");
  return ok();
}

// Codes and scales of a 4-bit matrix.
inline Checked check_mx4(const void* q, int64_t ldq, const void* s, int64_t lds, int64_t rows, int64_t cols) {
  if (rows == 0 || cols == 0) return ok();
  if (!q || !s) return fail(SFC_ERR_INVALID_ARG, "codes or scales are NULL");
  const int64_t blocks = mx4_blocks(cols);
  if (ldq < 16 * blocks) return fail(SFC_ERR_INVALID_ARG, "rows of codes are shorter than 16 bytes for every 32 values");
  if (lds < (blocks + 3) / 4 * 4)
    return fail(SFC_ERR_INVALID_ARG, "rows of scales are shorter than a byte for every 32 values, rounded up to 4");
  if ((uintptr_t)q % 16 || ldq % 16) return fail(SFC_ERR_UNSUPPORTED, "rows of codes must be 16-byte aligned");
  if ((uintptr_t)s % 4 || lds % 4) return fail(SFC_ERR_UNSUPPORTED, "rows of scales must be 4-byte aligned");
  if (ldq >= kMxMaxStride || lds >= kMxMaxStride)
    return fail(SFC_ERR_UNSUPPORTED, "rows of codes and scales must be less than 2^22 bytes apart");
  return ok();
}

inline Checked check_dims(int64_t a, int64_t b, int64_t c) {
  if (a < 0 || b < 0 || c < 0) return fail(SFC_ERR_INVALID_ARG, "sizes must be >= 0");
  if (a >= kMaxDim || b >= kMaxDim || c >= kMaxDim) return fail(SFC_ERR_UNSUPPORTED, "sizes must be < 2^31");
  return ok();
}

#define SFC_RETURN_IF(check)                        \
  do {                                              \
    const Checked checked_ = (check);               \
    if (checked_.code != SFC_OK) return checked_;   \
  } while (0)

inline Checked check_mx4_quant(int64_t rows, int64_t cols, const void* X, int64_t ldx, int type, const int32_t* order,
                               int64_t x_rows, int topk, const void* Q, int64_t ldq, const void* S, int64_t lds,
                               const void* Qt, int64_t ldqt, const void* St, int64_t ldst) {
  SFC_RETURN_IF(check_dims(rows, cols, order ? x_rows : 0));
  if (!type_ok(type)) return fail(SFC_ERR_INVALID_ARG, "unknown element type");
  if (order && topk < 1) return fail(SFC_ERR_INVALID_ARG, "topk must be >= 1");
  if (order && (uintptr_t)order % 4) return fail(SFC_ERR_UNSUPPORTED, "order is not aligned to its element size");
  if (rows == 0 || cols == 0) return ok();
  if ((Q == nullptr) != (S == nullptr) || (Qt == nullptr) != (St == nullptr))
    return fail(SFC_ERR_INVALID_ARG, "codes and scales go together");
  if (!Q && !Qt) return fail(SFC_ERR_INVALID_ARG, "no output");
  SFC_RETURN_IF(check_rows(X, order ? x_rows : rows, cols, ldx, type, "X is NULL", "ldx < cols"));
  if (Q) SFC_RETURN_IF(check_mx4(Q, ldq, S, lds, rows, cols));
  if (Qt) SFC_RETURN_IF(check_mx4(Qt, ldqt, St, ldst, cols, rows));
  return ok();
}

inline Checked check_mx4_dequant(int64_t rows, int64_t cols, const void* Q, int64_t ldq, const void* S, int64_t lds,
                                 const void* Y, int64_t ldy, int type) {
  SFC_RETURN_IF(check_dims(rows, cols, 0));
  if (!type_ok(type)) return fail(SFC_ERR_INVALID_ARG, "unknown element type");
  SFC_RETURN_IF(check_mx4(Q, ldq, S, lds, rows, cols));
  return check_rows(Y, rows, cols, ldy, type, "Y is NULL", "ldy < cols");
}

inline Checked check_blocks(int64_t M, int64_t N, int64_t groups) {
  if (ceil_div(M, 128) * ceil_div(N, 128) >= kMaxDim / (groups > 1 ? groups : 1))
    return fail(SFC_ERR_UNSUPPORTED, "too many output blocks");
  return ok();
}

// A caller's workspace (its size is checked against what the call's plan needs).
inline Checked check_workspace(const void* ws) {
  if ((uintptr_t)ws % 16) return fail(SFC_ERR_UNSUPPORTED, "workspace must be 16-byte aligned");
  return ok();
}

inline Checked check_gemm_mx4_sizes(int64_t M, int64_t N, int64_t K, int out_type) {
  SFC_RETURN_IF(check_dims(M, N, K));
  if (!type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown out_type");
  if (K % 32) return fail(SFC_ERR_INVALID_ARG, "K must be a multiple of 32");
  return ok();
}

inline Checked check_gemm_mx4(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* As, int64_t ldas,
                              const void* B, int64_t ldb, const void* Bs, int64_t ldbs, const void* C, int64_t ldc,
                              int out_type) {
  SFC_RETURN_IF(check_gemm_mx4_sizes(M, N, K, out_type));
  if (M == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(C, M, N, ldc, out_type, "C is NULL", "ldc < N"));
  SFC_RETURN_IF(check_mx4(A, lda, As, ldas, M, K));
  SFC_RETURN_IF(check_mx4(B, ldb, Bs, ldbs, N, K));
  return check_blocks(M, N, kAutoLayers);
}

inline Checked check_mx4_linear_sizes(int64_t M, int64_t N, int64_t K, int in_type, int out_type) {
  SFC_RETURN_IF(check_dims(M, N, K));
  if (!type_ok(in_type) || !type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown element type");
  return ok();
}

inline Checked check_mx4_linear(int64_t M, int64_t N, int64_t K, const void* X, int64_t ldx, int in_type, const void* W,
                                int64_t ldw, const void* Ws, int64_t ldws, const void* Y, int64_t ldy, int out_type) {
  SFC_RETURN_IF(check_mx4_linear_sizes(M, N, K, in_type, out_type));
  if (M == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(Y, M, N, ldy, out_type, "Y is NULL", "ldy < N"));
  SFC_RETURN_IF(check_rows(X, M, K, ldx, in_type, "X is NULL", "ldx < K"));
  SFC_RETURN_IF(check_mx4(W, ldw, Ws, ldws, N, K));
  if (16 * mx4_blocks(K) >= kMxMaxStride) return fail(SFC_ERR_UNSUPPORTED, "K must be below 2^23");
  return check_blocks(M, N, kAutoLayers);
}

inline Checked check_experts(int experts, int most) {
  if (experts < 1) return fail(SFC_ERR_INVALID_ARG, "experts must be >= 1");
  if (experts > most) return fail(SFC_ERR_UNSUPPORTED, "at most 1024 experts");
  return ok();
}

inline Checked check_index(const void* p, const char* null_text) {
  if (!p) return fail(SFC_ERR_INVALID_ARG, null_text);
  if ((uintptr_t)p % 4) return fail(SFC_ERR_UNSUPPORTED, "an index or weight array is not aligned to its element size");
  return ok();
}

inline Checked check_moe_gemm_mx4(int64_t rows, int64_t N, int64_t K, int experts, int most, const void* A, int64_t lda,
                                  const void* As, int64_t ldas, const void* B, int64_t ldb, int64_t stride_b,
                                  const void* Bs, int64_t ldbs, int64_t stride_bs, const void* offsets, const void* C,
                                  int64_t ldc, int out_type) {
  SFC_RETURN_IF(check_dims(rows, N, K));
  SFC_RETURN_IF(check_experts(experts, most));
  if (!type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown out_type");
  if (K % 32) return fail(SFC_ERR_INVALID_ARG, "K must be a multiple of 32");
  if (rows == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(C, rows, N, ldc, out_type, "C is NULL", "ldc < N"));
  SFC_RETURN_IF(check_index(offsets, "offsets is NULL"));
  SFC_RETURN_IF(check_mx4(A, lda, As, ldas, rows, K));
  SFC_RETURN_IF(check_mx4(B, ldb, Bs, ldbs, N, K));
  if (K > 0 && experts > 1) {
    if (stride_b < 0 || stride_bs < 0) return fail(SFC_ERR_INVALID_ARG, "the experts' strides must be >= 0");
    if (stride_b % 16 || stride_bs % 4)
      return fail(SFC_ERR_UNSUPPORTED, "the experts' strides must keep codes 16-byte and scales 4-byte aligned");
  }
  // a block of rows may be partly filled for every expert
  if ((ceil_div(rows, 128) + experts) * ceil_div(N, 16) >= kMaxDim || experts * ceil_div(N, 16) >= kMaxDim)
    return fail(SFC_ERR_UNSUPPORTED, "too many output blocks");
  return ok();
}

inline Checked check_moe_wgrad_mx4(int64_t M, int64_t N, int64_t rows, int experts, int most, const void* A, int64_t lda,
                                   const void* As, int64_t ldas, const void* B, int64_t ldb, const void* Bs,
                                   int64_t ldbs, const void* offsets, const void* C, int64_t ldc, int64_t stride_c,
                                   int out_type) {
  SFC_RETURN_IF(check_dims(M, N, rows));
  SFC_RETURN_IF(check_experts(experts, most));
  if (!type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown out_type");
  if (M == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(C, M, N, ldc, out_type, "C is NULL", "ldc < N"));
  if (experts > 1 && stride_c < 0) return fail(SFC_ERR_INVALID_ARG, "the stride between the experts' C must be >= 0");
  // one expert's matrix behind the other, or all experts' rows m before their rows m + 1
  if (experts > 1 && stride_c < (M - 1) * ldc + N && (stride_c < N || ldc < (experts - 1) * stride_c + N))
    return fail(SFC_ERR_INVALID_ARG, "the experts' C overlap");
  SFC_RETURN_IF(check_index(offsets, "offsets is NULL"));
  SFC_RETURN_IF(check_mx4(A, lda, As, ldas, M, rows));
  SFC_RETURN_IF(check_mx4(B, ldb, Bs, ldbs, N, rows));
  return check_blocks(M, N, experts);
}

inline Checked check_moe_sort(int64_t slots, int experts, int most, int align, const void* ids, int64_t rows,
                              const void* offsets, const void* order, const void* pos) {
  SFC_RETURN_IF(check_dims(slots, rows, 0));
  SFC_RETURN_IF(check_experts(experts, most));
  if (align < 1) return fail(SFC_ERR_INVALID_ARG, "align must be >= 1");
  if (align > (1 << 20)) return fail(SFC_ERR_UNSUPPORTED, "align must be at most 2^20");
  const int64_t need = slots + (int64_t)experts * (align - 1);
  if (need >= kMaxDim) return fail(SFC_ERR_UNSUPPORTED, "slots + experts * (align - 1) must be < 2^31");
  if (rows < need) return fail(SFC_ERR_INVALID_ARG, "rows < slots + experts * (align - 1)");
  SFC_RETURN_IF(check_index(offsets, "offsets is NULL"));
  if (rows > 0) SFC_RETURN_IF(check_index(order, "order is NULL"));
  if (slots > 0) SFC_RETURN_IF(check_index(ids, "the expert ids are NULL"));
  if (slots > 0) SFC_RETURN_IF(check_index(pos, "pos is NULL"));
  return ok();
}

// Sizes shared by dispatch, combine and its gradient.
inline Checked check_moe_sizes(int64_t tokens, int64_t rows, int64_t cols, int topk, int type) {
  SFC_RETURN_IF(check_dims(tokens, rows, cols));
  if (topk < 1) return fail(SFC_ERR_INVALID_ARG, "topk must be >= 1");
  if (!type_ok(type)) return fail(SFC_ERR_INVALID_ARG, "unknown element type");
  if (tokens * topk >= kMaxDim) return fail(SFC_ERR_UNSUPPORTED, "tokens * topk must be < 2^31");
  return ok();
}

inline Checked check_weights(const void* weights) {
  if ((uintptr_t)weights % 4)
    return fail(SFC_ERR_UNSUPPORTED, "an index or weight array is not aligned to its element size");
  return ok();
}

}  // namespace sfc
