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
  const __int128 matrix = (__int128)(rows - 1) * ld + cols, row = (__int128)(count - 1) * stride + cols;
  if (stride < matrix && (stride < cols || ld < row))
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
  if (order && K > 0 && a_rows * lda > kGatherMax)
    return fail(SFC_ERR_UNSUPPORTED, "rows taken through an order must lie within 2^31 elements");
  const bool nk = b_layout == SFC_B_NK;
  SFC_RETURN_IF(check_bf16(B, nk ? N : K, nk ? K : N, ldb, "B is NULL", "rows of B are longer than ldb"));
  if (K > 0 && experts > 1 && stride_b < 0) return fail(SFC_ERR_INVALID_ARG, "the experts' stride must be >= 0");
  // a block of rows may be partly filled for every expert
  if ((ceil_div(rows, 64) + experts) * ceil_div(N, 64) >= kMaxDim)
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
  if (ceil_div(M, 64) * ceil_div(N, 64) >= kMaxDim / experts) return fail(SFC_ERR_UNSUPPORTED, "too many output blocks");
  return ok();
}

// Sizes shared by the adapters' calls.
inline Checked check_lora_sizes(int64_t rows, int64_t cols, int64_t rank, int adapters, int most_rank, int layout) {
  SFC_RETURN_IF(check_dims(rows, cols, rank));
  SFC_RETURN_IF(check_layout(layout));
  if (adapters < 1) return fail(SFC_ERR_INVALID_ARG, "adapters must be >= 1");
  if (rank > most_rank) return fail(SFC_ERR_UNSUPPORTED, "ranks up to 256");
  return ok();
}

// Stacked weights of n x k (SFC_B_NK) or k x n.
inline Checked check_lora_weights(const void* W, int64_t n, int64_t k, int64_t ld, int64_t stride, int adapters, int layout) {
  const bool nk = layout == SFC_B_NK;
  SFC_RETURN_IF(check_rows(W, nk ? n : k, nk ? k : n, ld, SFC_OUT_BF16, "the adapters' weights are NULL",
                           "rows of the adapters' weights are longer than their leading dimension"));
  if (n > 0 && k > 0 && adapters > 1 && stride < 0) return fail(SFC_ERR_INVALID_ARG, "strides must be >= 0");
  return ok();
}

inline Checked check_lora_down(int64_t rows, int64_t K, int64_t rank, int adapters, int most_rank, const void* X, int64_t ldx,
                               const void* A, int64_t lda, int64_t stride_a, int layout, const void* ids, const void* scales,
                               const void* V, int64_t ldv) {
  SFC_RETURN_IF(check_lora_sizes(rows, K, rank, adapters, most_rank, layout));
  if (rows == 0 || rank == 0) return ok();
  SFC_RETURN_IF(check_rows(V, rows, rank, ldv, SFC_OUT_F32, "V is NULL", "ldv < rank"));
  SFC_RETURN_IF(check_bf16(X, rows, K, ldx, "X is NULL", "ldx < K"));
  if (K > 0 && lda >= kRowsMaxLd)
    return fail(SFC_ERR_UNSUPPORTED, "leading dimensions of bf16 operands must be below 2^22");
  SFC_RETURN_IF(check_lora_weights(A, rank, K, lda, stride_a, adapters, layout));
  SFC_RETURN_IF(check_weights(scales));
  return check_index(ids, "ids is NULL");
}

inline Checked check_lora_up(int64_t rows, int64_t N, int64_t rank, int adapters, int most_rank, const void* V, int64_t ldv,
                             const void* B, int64_t ldb, int64_t stride_b, int layout, const void* ids, const void* base,
                             int64_t ld_base, const void* Y, int64_t ldy, int type) {
  SFC_RETURN_IF(check_lora_sizes(rows, N, rank, adapters, most_rank, layout));
  if (!type_ok(type)) return fail(SFC_ERR_INVALID_ARG, "unknown element type");
  if (rows == 0 || N == 0) return ok();
  SFC_RETURN_IF(check_rows(Y, rows, N, ldy, type, "Y is NULL", "ldy < N"));
  if (base) SFC_RETURN_IF(check_rows(base, rows, N, ld_base, type, "", "ld_base < N"));
  if (base == Y && ld_base != ldy) return fail(SFC_ERR_INVALID_ARG, "base may be Y, but not lie across it");
  SFC_RETURN_IF(check_rows(V, rows, rank, ldv, SFC_OUT_F32, "V is NULL", "ldv < rank"));
  SFC_RETURN_IF(check_lora_weights(B, N, rank, ldb, stride_b, adapters, layout));
  return check_index(ids, "ids is NULL");
}

inline Checked check_lora_wgrad(int64_t rows, int64_t cols, int64_t rank, int adapters, int most_rank, const void* Z,
                                int64_t ldz, const void* V, int64_t ldv, const void* ids, const void* G, int64_t ldg,
                                int64_t stride_g, int layout, int out_type) {
  SFC_RETURN_IF(check_lora_sizes(rows, cols, rank, adapters, most_rank, layout));
  if (!type_ok(out_type)) return fail(SFC_ERR_INVALID_ARG, "unknown out_type");
  if (cols == 0 || rank == 0) return ok();
  const bool nk = layout == SFC_B_NK;
  const int64_t r = nk ? cols : rank, c = nk ? rank : cols;
  SFC_RETURN_IF(check_rows(G, r, c, ldg, out_type, "G is NULL", "rows of G are longer than ldg"));
  SFC_RETURN_IF(check_stack(r, c, ldg, adapters, stride_g, "the adapters' G overlap"));
  SFC_RETURN_IF(check_rows(Z, rows, cols, ldz, SFC_OUT_BF16, "Z is NULL", "ldz < columns"));
  SFC_RETURN_IF(check_rows(V, rows, rank, ldv, SFC_OUT_F32, "V is NULL", "ldv < rank"));
  if (rows > 0) SFC_RETURN_IF(check_index(ids, "ids is NULL"));
  return ok();
}

}  // namespace sfc
