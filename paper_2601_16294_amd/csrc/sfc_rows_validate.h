// Argument checks of the bf16 expert and adapter entry points, free of any HIP dependency; every
// check happens before the library touches the device.
#pragma once
#include "sfc_ops_validate.h"

namespace sfc {

constexpr int64_t kRowsMaxLd = (int64_t)1 << 22;      // elements: 256 rows stay within 32-bit offsets
constexpr int64_t kGatherMax = ((int64_t)1 << 31) - (1 << 11);    // elements reached through an order

inline Checked check_layout(int layout) {
  if (layout != SFC_B_NK && layout != SFC_B_KN) return fail(SFC_ERR_INVALID_ARG, "unknown layout of B");
  return ok();
}

inline Checked check_bf16(const void* p, int64_t rows, int64_t cols, int64_t ld, const char* null_text, const char* ld_text) {
  SFC_RETURN_IF(check_rows(p, rows, cols, ld, SFC_OUT_BF16, null_text, ld_text));
  if (rows > 0 && cols > 0 && ld >= kRowsMaxLd)
    return fail(SFC_ERR_UNSUPPORTED, "leading dimensions of bf16 operands must be below 2^22");
  return ok();
}

// `count` outputs of rows x cols, `stride` elements apart, that must not overlap: they lie one behind
// the other, or their rows in turn.
inline Checked check_stack(int64_t rows, int64_t cols, int64_t ld, int64_t count, int64_t stride, const char* overlap_text) {
  if (count < 2) return ok();
  if (stride < 0) return fail(SFC_ERR_INVALID_ARG, "strides must be >= 0");
  if (stride < (rows - 1) * ld + cols && (stride < cols || ld < (count - 1) * stride + cols))
    return fail(SFC_ERR_INVALID_ARG, overlap_text);
  return ok();
}

inline Checked check_moe_gemm(int64_t rows, int64_t N, int64_t K, int experts, int most, const void* A, int64_t lda,
                              const void* order, int64_t a_rows, int topk, const void* B, int64_t ldb, int64_t stride_b,
                              int b_layout, const void* offsets, const void* C, int64_t ldc, int out_type) {
  SFC_RETURN_IF(check_dims(rows, N, K));
  SFC_RETURN_IF(check_experts(experts, most));
  SFC_RETURN_IF(check_layout(b_layout));
  if (!type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown out_type");
  if (order) {
    SFC_RETURN_IF(check_dims(a_rows, 0, 0));
    if (topk < 1) return fail(SFC_ERR_INVALID_ARG, "topk must be >= 1");
  }
  if (rows == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(C, rows, N, ldc, out_type, "C is NULL", "ldc < N"));
  SFC_RETURN_IF(check_index(offsets, "offsets is NULL"));
  if (order) SFC_RETURN_IF(check_index(order, "order is NULL"));
  SFC_RETURN_IF(check_bf16(A, order ? a_rows : rows, K, lda, "A is NULL", "lda < K"));
  if (order && a_rows * lda > kGatherMax)
    return fail(SFC_ERR_UNSUPPORTED, "rows taken through an order must lie within 2^31 elements");
  const bool nk = b_layout == SFC_B_NK;
  SFC_RETURN_IF(check_bf16(B, nk ? N : K, nk ? K : N, ldb, "B is NULL", "rows of B are longer than ldb"));
  if (K > 0 && experts > 1 && stride_b < 0) return fail(SFC_ERR_INVALID_ARG, "the experts' stride must be >= 0");
  // a block of rows may be partly filled for every expert
  if ((ceil_div(rows, 128) + experts) * ceil_div(N, 16) >= kMaxDim)
    return fail(SFC_ERR_UNSUPPORTED, "too many output blocks");
  return ok();
}

inline Checked check_moe_wgrad(int64_t M, int64_t N, int64_t rows, int experts, int most, const void* A, int64_t lda,
                               const void* B, int64_t ldb, const void* offsets, const void* C, int64_t ldc,
                               int64_t stride_c, int out_type) {
  SFC_RETURN_IF(check_dims(M, N, rows));
  SFC_RETURN_IF(check_experts(experts, most));
  if (!type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown out_type");
  if (M == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(C, M, N, ldc, out_type, "C is NULL", "ldc < N"));
  SFC_RETURN_IF(check_stack(M, N, ldc, experts, stride_c, "the experts' C overlap"));
  SFC_RETURN_IF(check_index(offsets, "offsets is NULL"));
  SFC_RETURN_IF(check_bf16(A, rows, M, lda, "A is NULL", "lda < M"));
  SFC_RETURN_IF(check_bf16(B, rows, N, ldb, "B is NULL", "ldb < N"));
  return check_blocks(M, N, experts);
}

}  // namespace sfc
